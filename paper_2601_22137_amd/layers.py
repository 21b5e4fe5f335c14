"""The layer operators for autograd, and the attention half of a transformer layer made of them: the part of a model whose 2-D weights
optim.muon_orthogonalize updates.

Every step of the operators, gradients included, runs in the HIP kernels; the projections are PyTorch products.  Second derivatives of attention and of norm and rotation are an error.
"""
import torch
from torch.autograd.function import once_differentiable

from . import prism


# Tensors of the masks and positions are arguments of their own: written to between the passes, they are an error as other saved tensors are.

class _NormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, inv_freq, positions, options):
        ctx.save_for_backward(q, k, q_weight, k_weight, inv_freq, positions)
        ctx.options = options
        return prism.qk_norm_rope(q, k, q_weight=q_weight, k_weight=k_weight, inv_freq=inv_freq, positions=positions, **options)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq_out, dk_out):
        q, k, q_weight, k_weight, inv_freq, positions = ctx.saved_tensors
        # the gradient of a result that nothing reads is None, and so is that of one that there is not
        dq_out, dk_out = (_rows(g) if g is not None else None if t is None else torch.zeros_like(t) for g, t in ((dq_out, q), (dk_out, k)))
        dq, dk, dqw, dkw = prism.qk_norm_rope_backward(dq_out, dk_out, q, k, q_weight=q_weight, k_weight=k_weight, inv_freq=inv_freq, positions=positions, **ctx.options)
        return dq, dk, dqw if q_weight is not None else None, dkw if k_weight is not None else None, None, None, None


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, slopes, prefix, k_lens, q_doc, k_doc, options):
        masks = dict(slopes=slopes, prefix=prefix, k_lens=k_lens, q_doc=q_doc, k_doc=k_doc)
        out, lse = prism.attention(q, k, v, **masks, **options)
        ctx.save_for_backward(q, k, v, out, lse, *masks.values())
        ctx.options = options
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        q, k, v, out, lse, slopes, prefix, k_lens, q_doc, k_doc = ctx.saved_tensors
        return prism.attention_backward(_rows(dout), q, k, v, out, lse, slopes=slopes, prefix=prefix, k_lens=k_lens, q_doc=q_doc, k_doc=k_doc, **ctx.options) + 6 * (None,)


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, seed, offset):
        ctx.args = p, seed, offset
        return prism.dropout(x, p, seed, offset=offset, residual=residual)

    @staticmethod
    def backward(ctx, dy):
        # the same call, so that derivatives of the gradient are right too
        dx = _Dropout.apply(dy.contiguous(), None, *ctx.args) if ctx.needs_input_grad[0] else None
        return dx, dy if ctx.needs_input_grad[1] else None, None, None, None


def _rows(t):
    """The entries of every head next to each other (autograd hands out expanded gradients)."""
    return t if t.stride(3) == 1 or t.shape[3] == 1 else t.contiguous()


def _fixed(t, name):
    if t is not None and t.requires_grad and torch.is_grad_enabled():
        raise prism.PrismError("%s: there is no gradient for it" % name)


def norm_rope(q, k, q_weight=None, k_weight=None, inv_freq=None, positions=None, start=0, norm=True, interleaved=False, scale=1.0, eps=1e-6):
    """prism.qk_norm_rope of queries and keys (or of one of them) with gradients for them and the weights."""
    _fixed(inv_freq, "inv_freq")
    options = dict(start=start, norm=norm, interleaved=interleaved, scale=scale, eps=eps)
    if not torch.is_grad_enabled():       # tokens one by one: the host's time counts
        return prism.qk_norm_rope(q, k, q_weight=q_weight, k_weight=k_weight, inv_freq=inv_freq, positions=positions, **options)
    return _NormRope.apply(q, k, q_weight, k_weight, inv_freq, positions, options)


def attention(q, k, v, scale=None, causal=False, softcap=0.0, slopes=None, prefix=None, k_lens=None, q_doc=None, k_doc=None, workspace=None):
    """prism.attention with gradients for q, k and v.  A workspace has to be enough for the gradients too."""
    _fixed(slopes, "slopes")
    return _Attention.apply(q, k, v, slopes, prefix, k_lens, q_doc, k_doc, dict(scale=scale, causal=causal, softcap=softcap, workspace=workspace))


def dropout(x, p, seed, offset=0, residual=None):
    """prism.dropout with gradients for x and the residual."""
    return _Dropout.apply(x.contiguous(), None if residual is None else residual.contiguous(), p, seed, offset)


def _capturing(t):
    return t.is_cuda and torch.cuda.is_current_stream_capturing()


class Cache(tuple):
    """(keys, values, lens): [batch, length, k_heads, dim] twice, and how many tokens there are of each sequence, int32 on the device.  How many the longest has is
    also known on the host; it is read from the device only after lens was written to by others, or by a step that was captured into a graph."""

    def __new__(cls, keys, values, lens):
        self = tuple.__new__(cls, (keys, values, lens))
        self.longest, self.version, self.captured = 0, None, False
        self.rows = torch.arange(lens.shape[0], device=lens.device)
        return self

    def __getnewargs__(self):          # copies and pickles
        return tuple(self)

    def _written(self):
        """Changes with every write to lens (tensors of inference mode do not tell)."""
        lens = self[2]
        return 0 if lens.is_inference() else lens._version

    def _read(self):
        lens = self[2]
        return int(lens.max()) if lens.numel() else 0

    def last_place(self):
        """Index of the last token there is room for; an error, before anything is written, if it is taken."""
        keys, _, lens = self
        if _capturing(lens):
            self.captured = True
        else:
            if self.captured or self.version != self._written():
                self.longest = self._read()
            if self.longest >= keys.shape[1]:
                raise prism.PrismError("the cache is full: it is made for %d tokens" % keys.shape[1])
        return keys.shape[1] - 1

    def took_one(self):
        self.longest += 1
        self.version = self._written()


class SelfAttention(torch.nn.Module):
    """x + dropout(attention(x w_qkv) w_out): one projection for queries, keys and values, whose parts are used as views; norms of the heads of queries and
    keys, rotation by position (of their first rot_dim entries; None: all), scores capped at will; queries in groups of heads / k_heads share a key head."""

    def __init__(self, width, heads, k_heads=None, head_dim=None, rot_dim=None, softcap=0.0, p=0.0, base=10000.0, dtype=torch.bfloat16, device="cuda"):
        super().__init__()
        self.heads, self.k_heads, self.dim = heads, k_heads or heads, head_dim or width // heads
        self.softcap, self.p = softcap, p
        inner = (self.heads + 2 * self.k_heads) * self.dim
        self.w_qkv = torch.nn.Parameter(torch.randn(inner, width, dtype=dtype, device=device) * width ** -0.5)
        self.w_out = torch.nn.Parameter(torch.randn(width, self.heads * self.dim, dtype=dtype, device=device) * (self.heads * self.dim) ** -0.5)
        self.q_weight = torch.nn.Parameter(torch.ones(self.dim, device=device))
        self.k_weight = torch.nn.Parameter(torch.ones(self.dim, device=device))
        rot_dim = self.dim if rot_dim is None else rot_dim
        inv_freq, self.rope_scale = prism.rope_frequencies(rot_dim, base=base, device=device) if rot_dim else (None, 1.0)
        self.register_buffer("inv_freq", inv_freq, persistent=False)

    def _project(self, x, positions):
        b, n, _ = x.shape
        hq, hk, d = self.heads, self.k_heads, self.dim
        q, k, v = (x @ self.w_qkv.t()).view(b, n, hq + 2 * hk, d).split([hq, hk, hk], dim=2)
        q, k = norm_rope(q, k, self.q_weight, self.k_weight, inv_freq=self.inv_freq, positions=positions, scale=self.rope_scale)
        return q, k, v

    def forward(self, x, positions=None, doc=None, seed=None, offset=None):
        """x [batch, token, width]; positions and documents int32 [batch, token] (a negative document is padding).  Seed and offset name the mask of the dropout; without
        either, one is drawn from PyTorch's generator of the host."""
        b, n, _ = x.shape
        q, k, v = self._project(x, positions)
        y = attention(q, k, v, causal=True, softcap=self.softcap, q_doc=doc, k_doc=doc).reshape(b, n, -1) @ self.w_out.t()
        p = self.p if self.training else 0.0
        if p > 0.0 and seed is None and offset is None:
            seed = int(torch.randint(2 ** 63 - 1, (), device="cpu"))
        return dropout(y, p, seed or 0, offset or 0, residual=x)

    def new_cache(self, batch, length):
        """Keys and values of up to `length` tokens, and how many there are of each sequence."""
        make = lambda: torch.zeros(batch, length, self.k_heads, self.dim, dtype=self.w_qkv.dtype, device=self.w_qkv.device)   # noqa: E731
        cache = Cache(make(), make(), torch.zeros(batch, dtype=torch.int32, device=self.w_qkv.device))
        cache.version = cache._written()
        return cache

    @torch.no_grad()
    def step(self, x, cache):
        """One token of each sequence, x [batch, 1, width], behind the tokens in the cache, which takes it in.  (How often a step that is captured into a graph is
        replayed is the caller's to count: tokens too many then replace the last one.)"""
        if not isinstance(cache, Cache):
            cache = Cache(*cache)
        last = cache.last_place()
        keys, values, lens = cache
        b = x.shape[0]
        q, k, v = self._project(x, lens.view(b, 1))
        at = cache.rows, lens.clamp(0, last).long()
        keys[at], values[at] = k[:, 0], v[:, 0]
        lens += 1
        cache.took_one()
        out, _ = prism.attention(q, keys, values, softcap=self.softcap, k_lens=lens)
        return x + out.reshape(b, 1, -1) @ self.w_out.t()
