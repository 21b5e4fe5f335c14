"""The operators at the ends of a model: the library's checks and workspace sizes, and how layers.py hands gradients on.  Nothing here needs a GPU: pointers are never read (every call is
refused, or empty, before anything is enqueued), and the calls under autograd are stand-ins."""
import ctypes
import os

import pytest
import torch

ADDRESS = 1 << 20


@pytest.fixture(scope="module")
def prism():
    from paper_2601_22137_amd import build, prism as P
    if not os.path.exists(P.LIB_PATH):
        build.build(verbose=False)
    P.lib()
    return P


def _desc(kind, **kw):
    d = kind()
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _embedding(prism, **kw):
    return _desc(prism.EmbeddingDesc, **dict(dict(count=10, rows=20, width=8, scale=1.0, table_stride=8, out_stride=8), **kw))


def _norm(prism, **kw):
    return _desc(prism.LayerNormDesc, **dict(dict(rows=10, width=8, eps=1e-5, x=8, residual=8, total=8, y=8, dy=8, dtotal=8, dx=8), **kw))


def _logits(prism, **kw):
    return _desc(prism.LogitsDesc, **dict(dict(rows=10, vocabulary=8, scale=1.0, logits_stride=8, dlogits_stride=8, clip_low=0.2, clip_high=0.2), **kw))


@pytest.mark.parametrize("kw,rc", [(dict(count=-1), "EINVAL"), (dict(rows=-1), "EINVAL"), (dict(width=0), "EINVAL"), (dict(scale=float("nan")), "EINVAL"), (dict(table_stride=-8), "EINVAL"),
                                   (dict(out_stride=-1), "EINVAL"), (dict(out_stride=1 << 60), "EINVAL"), (dict(count=(1 << 30) + 1), "EUNSUPPORTED"), (dict(rows=(1 << 27) + 1), "EUNSUPPORTED")])
def test_embedding_refuses(prism, kw, rc):
    L, d = prism.lib(), _embedding(prism, **kw)
    for call in (L.prism_embedding, L.prism_embedding_backward):
        assert call(ADDRESS, ADDRESS, ADDRESS, prism.BF16, ctypes.byref(d), None) == getattr(prism, rc)
        assert L.prism_last_error()
    out = ctypes.c_size_t(0)
    assert L.prism_embedding_workspace_bytes(prism.F32, ctypes.byref(d), ctypes.byref(out)) == getattr(prism, rc)


@pytest.mark.parametrize("kw", [dict(rows=-1), dict(width=0), dict(eps=-1.0), dict(eps=float("inf")), dict(x=-1), dict(dx=-8), dict(dtotal=1 << 60)])
def test_layer_norm_refuses(prism, kw):
    L, d = prism.lib(), _norm(prism, **kw)
    assert L.prism_layer_norm(*[ADDRESS] * 5, ADDRESS + 64, ADDRESS, prism.F32, ctypes.byref(d), None) == prism.EINVAL
    assert L.prism_layer_norm_backward(*[ADDRESS] * 8, prism.F32, ctypes.byref(d), None) == prism.EINVAL
    assert L.prism_layer_norm_workspace_bytes(prism.F32, ctypes.byref(d), ctypes.byref(ctypes.c_size_t(0))) == prism.EINVAL


@pytest.mark.parametrize("kw", [dict(rows=-1), dict(vocabulary=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=1e-60), dict(scale=1e-31), dict(scale=2e30), dict(scale=3e38), dict(logits_stride=-1),
                                dict(dlogits_stride=-8)])
def test_logits_refuse(prism, kw):
    L, d = prism.lib(), _logits(prism, **kw)
    assert L.prism_token_logprob(*[ADDRESS] * 4, prism.BF16, ctypes.byref(d), None) == prism.EINVAL
    assert L.prism_token_logprob_backward(*[ADDRESS] * 5, prism.BF16, ctypes.byref(d), None) == prism.EINVAL
    assert L.prism_policy_loss(*[ADDRESS] * 7, prism.BF16, ctypes.byref(d), None) == prism.EINVAL
    assert L.prism_policy_loss_workspace_bytes(ctypes.byref(d), ctypes.byref(ctypes.c_size_t(0))) == prism.EINVAL


@pytest.mark.parametrize("kw", [dict(clip_low=-0.1), dict(clip_low=1.1), dict(clip_high=-0.1), dict(clip_high=float("inf")), dict(kl=-1.0), dict(kl=float("nan")), dict(kl=0.1)])
def test_policy_loss_refuses(prism, kw):
    assert prism.lib().prism_policy_loss(*[ADDRESS] * 7, prism.BF16, ctypes.byref(_logits(prism, **kw)), None) == prism.EINVAL


def test_pointers_sizes_and_overlaps(prism):
    L, A = prism.lib(), ADDRESS
    e, n, z = (ctypes.byref(f(prism)) for f in (_embedding, _norm, _logits))
    for call, count, desc in ((L.prism_embedding, 3, e), (L.prism_embedding_backward, 3, e), (L.prism_token_logprob_backward, 5, z)):
        for i in range(count):
            for bad in (None, A + 1):
                args = [A] * count
                args[i] = bad
                assert call(*args, prism.BF16, desc, None) == prism.EINVAL, (call, i)
        assert call(*[A] * count, 9, desc, None) == prism.EINVAL and call(*[A] * count, prism.F32, None, None) == prism.EINVAL
    B = A + 4096
    for args in ((None, A, A, A, A, B, A), (A, A, A, A, None, B, A), (A, None, A, A, A, B, A), (A, A, A, A, A, None, A), (A, A, A, A, A, A, A), (A, A, A + 2, A, A, B, A), (A, A, A, A, A, B, A + 4)):
        assert L.prism_layer_norm(*args, prism.F32, n, None) == prism.EINVAL, args
    for i in (0, 1, 2, 5):
        args = [A] * 8
        args[i] = None
        assert L.prism_layer_norm_backward(*args, prism.F32, n, None) == prism.EINVAL
    for args in ((None, A, A, A, A, A, A), (A, None, A, A, A, A, A), (A, A, None, A, A, A, A), (A, A, A, A + 2, A, A, A), (A, A, A, A, A, A, A + 1)):
        assert L.prism_policy_loss(*args, prism.F32, z, None) == prism.EINVAL
    # rows of results over one another
    assert L.prism_embedding(A, A, A, prism.F32, ctypes.byref(_embedding(prism, out_stride=7)), None) == prism.EINVAL
    assert L.prism_embedding_backward(A, A, A, prism.F32, ctypes.byref(_embedding(prism, table_stride=0)), None) == prism.EINVAL
    assert L.prism_layer_norm(A, A, A, A, A, B, A, prism.F32, ctypes.byref(_norm(prism, y=4)), None) == prism.EINVAL
    assert L.prism_layer_norm_backward(*[A] * 8, prism.F32, ctypes.byref(_norm(prism, dx=4)), None) == prism.EINVAL
    assert L.prism_policy_loss(*[A] * 7, prism.F32, ctypes.byref(_logits(prism, dlogits_stride=7)), None) == prism.EINVAL
    # sizes
    assert L.prism_layer_norm(A, A, A, A, A, B, A, prism.F32, ctypes.byref(_norm(prism, width=prism_max(prism) + 1)), None) == prism.EUNSUPPORTED
    assert L.prism_token_logprob(A, A, A, A, prism.F32, ctypes.byref(_logits(prism, rows=1 << 31, logits_stride=1)), None) == prism.EUNSUPPORTED


def prism_max(prism):
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "prism.h")).read()
    return int(header.split("#define PRISM_MAX_NORM_WIDTH")[1].split()[0])


def test_empty_calls_touch_nothing(prism):
    L = prism.lib()
    assert L.prism_embedding(None, None, None, prism.F32, ctypes.byref(_embedding(prism, count=0)), None) == prism.OK
    assert L.prism_embedding_backward(None, None, None, prism.F32, ctypes.byref(_embedding(prism, rows=0)), None) == prism.OK
    assert L.prism_layer_norm(*[None] * 7, prism.F32, ctypes.byref(_norm(prism, rows=0)), None) == prism.OK
    assert L.prism_layer_norm_backward(*[None] * 8, prism.F32, ctypes.byref(_norm(prism, rows=0)), None) == prism.OK
    assert L.prism_token_logprob(*[None] * 4, prism.F32, ctypes.byref(_logits(prism, rows=0)), None) == prism.OK
    assert L.prism_token_logprob_backward(*[None] * 5, prism.F32, ctypes.byref(_logits(prism, rows=0)), None) == prism.OK


def test_workspaces(prism):
    L, out = prism.lib(), ctypes.c_size_t(0)
    for count, rows, width in ((1, 1, 1), (65536, 32768, 768), (100, 131072, 4096), (1 << 22, 1000, 8192), (1 << 30, 10, 1)):
        d = _embedding(prism, count=count, rows=rows, width=width, table_stride=width, out_stride=width)
        assert L.prism_embedding_workspace_bytes(prism.BF16, ctypes.byref(d), ctypes.byref(out)) == prism.OK
        # starts, sorted tokens, and two rows of sums for four tokens at most, padded to 512 columns
        assert 4 * rows + 8 * count <= out.value <= 4 * (rows + 1) + 8 * count + (count // 4 + 1) * 2 * (width + 512) * 4 + 1024
    for rows, width in ((1, 1), (65536, 768), (8, 16384)):
        d = _norm(prism, rows=rows, width=width)
        assert L.prism_layer_norm_workspace_bytes(prism.F32, ctypes.byref(d), ctypes.byref(out)) == prism.OK and out.value <= 1024 * 2 * width * 4 + 256
    assert L.prism_policy_loss_workspace_bytes(ctypes.byref(_logits(prism, rows=1000)), ctypes.byref(out)) == prism.OK and 8000 < out.value < 9000


def test_descriptions_are_packed_as_the_header_says(prism):
    for layout, kind in ((prism._EMBEDDING, prism.EmbeddingDesc), (prism._LAYER_NORM, prism.LayerNormDesc), (prism._LOGITS, prism.LogitsDesc)):
        assert layout.size == ctypes.sizeof(kind)
        fields = [f for f, _ in kind._fields_]
        d = kind.from_buffer_copy(layout.pack(*range(1, len(fields) + 1)))
        assert [getattr(d, f) for f in fields] == list(range(1, len(fields) + 1))


# ---- under autograd

@pytest.fixture
def layers(prism, monkeypatch):
    """Calls of the right shapes that need no GPU: gradients keep a trace of what they were made from."""
    from paper_2601_22137_amd import layers as M

    def embedding(tokens, table, scale=1.0):
        assert tokens.is_contiguous()
        return table[tokens] * scale

    def embedding_backward(dout, tokens, rows, scale=1.0):
        assert dout.is_contiguous()
        return torch.zeros(rows, dout.shape[-1]).index_add_(0, tokens.flatten(), dout.flatten(0, -2)) * scale

    def layer_norm(x, weight, bias, residual=None, center=True, eps=1e-5):
        total = x if residual is None else x + residual
        return 2 * total, total, torch.zeros(x.numel() // x.shape[-1], 2)

    def layer_norm_backward(dy, total, stats, weight=None, dtotal=None, center=True, bias=True):
        assert dy.is_contiguous() and (dtotal is None or dtotal.is_contiguous())
        return 2 * dy + (0 if dtotal is None else dtotal), dy.flatten(0, -2).sum(0), dy.flatten(0, -2).sum(0) * 3 if bias else None

    def token_logprob(logits, tokens, scale=1.0):
        return scale * logits.gather(-1, tokens.unsqueeze(-1)).squeeze(-1), torch.zeros(tokens.shape)

    def token_logprob_backward(dlogp, logits, tokens, lse, scale=1.0):
        assert dlogp.is_contiguous()
        return torch.zeros_like(logits).scatter(-1, tokens.unsqueeze(-1), dlogp.unsqueeze(-1) * scale)

    def policy_loss(logits, tokens, advantages=None, old_logp=None, ref_logp=None, weights=None, clip=(0.2, 0.2), kl=0.0, scale=1.0, gradient=True):
        assert not gradient and all(t is None or t.is_contiguous() for t in (tokens, advantages, old_logp, ref_logp, weights))
        logp, lse = token_logprob(logits, tokens, scale)
        return prism.PolicyLoss(-logp.sum(), logp, lse, torch.full_like(logp, -1.0), None)
    for f in (embedding, embedding_backward, layer_norm, layer_norm_backward, token_logprob, token_logprob_backward, policy_loss):
        monkeypatch.setattr(prism, f.__name__, torch.no_grad()(f))
    return M


def test_embedding_gradient(layers):
    table, tokens = torch.randn(5, 3, requires_grad=True), torch.tensor([[1, 2, 0], [1, 1, 4]]).t()        # not contiguous
    layers.embedding(tokens, table, scale=2.0).sum().backward()                                             # the gradient comes expanded
    assert torch.equal(table.grad, torch.tensor([2.0, 6.0, 2.0, 0.0, 2.0]).view(5, 1).expand(5, 3))
    y = layers.embedding(tokens := tokens.contiguous(), table)
    tokens.zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_layer_norm_gradients(layers):
    x, r, w, b = torch.randn(2, 3, 4, requires_grad=True), torch.randn(2, 3, 4, requires_grad=True), torch.ones(4, requires_grad=True), torch.ones(4, requires_grad=True)
    y, total = layers.layer_norm(x, w, b, residual=r)
    (y.sum() + (5 * total).sum()).backward()
    assert torch.all(x.grad == 7) and torch.all(r.grad == 7) and torch.all(w.grad == 6) and torch.all(b.grad == 18)
    for pick, gx, gw in ((0, 2, 6), (1, 1, 0)):               # one of the two results only
        x.grad = w.grad = None
        layers.layer_norm(x, w, b, residual=r)[pick].sum().backward()
        assert torch.all(x.grad == gx) and torch.all(w.grad == gw)
    x.grad = w.grad = None
    layers.layer_norm(x).sum().backward()
    assert torch.all(x.grad == 2)
    with torch.no_grad():
        assert torch.is_tensor(layers.layer_norm(x)) and len(layers.layer_norm(x, residual=r)) == 2


def test_losses_and_gradients(layers):
    z, t = torch.randn(2, 3, 7, requires_grad=True), torch.tensor([[1, 2, 0], [1, 1, 4]])
    one = torch.zeros(2, 3, 7).scatter(-1, t.unsqueeze(-1), 1.0)
    layers.token_logprob(z, t, scale=0.5).sum().backward()
    assert torch.equal(z.grad, 0.5 * one)
    z.grad = None
    loss, logp = layers.policy_loss(z, t.t().contiguous().t(), scale=0.5, weights=torch.ones(3, 2).t())
    assert not logp.requires_grad
    (3 * loss).backward()
    assert torch.equal(z.grad, -1.5 * one)


def test_what_has_no_gradient_is_refused(layers, prism):
    z, t = torch.randn(3, 7, requires_grad=True), torch.tensor([1, 2, 0])
    learned = torch.zeros(3, requires_grad=True)
    for name in ("advantages", "old_logp", "ref_logp", "weights"):
        with pytest.raises(prism.PrismError, match=name):
            layers.policy_loss(z, t, **{name: learned})
    (g,) = torch.autograd.grad((layers.token_logprob(z, t) ** 2).sum(), z, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.sum().backward()


def test_modules(layers):
    e, n, rms = layers.Embedding(9, 4, scale=2.0, dtype=torch.float32, device="cpu"), layers.LayerNorm(4, device="cpu"), layers.LayerNorm(4, center=False, device="cpu")
    assert {k for k, _ in n.named_parameters()} == {"weight", "bias"} and [k for k, _ in rms.named_parameters()] == ["weight"]
    x = e(torch.tensor([[1, 8]]))
    y, total = rms(*([n(x)] * 2))
    (y.sum() + total.sum()).backward()
    assert e.weight.grad is not None and n.bias.grad is not None and rms.weight.grad is not None
