"""The operators at the ends of a model under autograd and together: gradients against PyTorch's in 64 bits and against differences, a training step of a small model, eagerly and
captured, and the example's policy step."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
V, W, ROWS = 300, 72, 50


@pytest.fixture(scope="module")
def layers():
    from paper_2601_22137_amd import layers as M, prism
    prism.lib()
    return M


def _inputs(seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g).cuda()   # noqa: E731
    tokens = torch.randint(-1, V, (ROWS,), generator=g).cuda()
    targets = torch.randint(-1, V, (ROWS,), generator=g).cuda()
    params = dict(table=r(V, W), w1=1 + 0.2 * r(W), b1=r(W), w2=1 + 0.2 * r(W))
    given = dict(advantages=r(ROWS), old_logp=-5 + 0.2 * r(ROWS), ref_logp=-5 + 0.2 * r(ROWS), weights=torch.rand(ROWS, generator=g).cuda() / ROWS)
    return tokens, targets, params, given


def _model(L, tokens, targets, p, given):
    """Embedding, a norm, its sum with the embedding through a second norm, logits by the table, loss; and a part that reads the stream and the log-probabilities directly."""
    x = L.embedding(tokens, p["table"], scale=0.5)
    a = L.layer_norm(x, p["w1"], p["b1"])
    y, total = L.layer_norm(a, p["w2"], residual=x, center=False)
    z = y @ p["table"].t()
    loss, _ = L.policy_loss(z, targets, kl=0.1, scale=0.3, **given)
    return loss + 1e-3 * total.square().mean() - 0.1 * L.token_logprob(z, targets, scale=0.3).mean()


class _Plain:
    """The same from elementary operations."""
    @staticmethod
    def embedding(tokens, table, scale):
        return torch.where((tokens >= 0).unsqueeze(1), table[tokens.clamp(min=0)] * scale, torch.zeros((), dtype=table.dtype, device="cuda"))

    @staticmethod
    def layer_norm(x, w, b=None, residual=None, center=True):
        h = x if residual is None else x + residual
        d = h - h.mean(-1, keepdim=True) if center else h
        y = d / torch.sqrt((d * d).mean(-1, keepdim=True) + 1e-5) * w + (0 if b is None else b)
        return y if residual is None else (y, h)

    @staticmethod
    def token_logprob(z, t, scale):
        a = z * scale
        return torch.where(t >= 0, a.gather(1, t.clamp(min=0).unsqueeze(1)).squeeze(1) - torch.logsumexp(a, 1), torch.zeros((), dtype=z.dtype, device="cuda"))

    @classmethod
    def policy_loss(cls, z, t, advantages, old_logp, ref_logp, weights, kl, scale):
        logp = cls.token_logprob(z, t, scale)
        r, f = torch.exp(logp - old_logp), ref_logp - logp
        l = -torch.minimum(r * advantages, r.clamp(0.8, 1.2) * advantages) + kl * (torch.exp(f) - f - 1)
        return (torch.where(t >= 0, weights, torch.zeros_like(weights)) * l).sum(), logp


def _off_the_edges(given, tokens, targets, params):
    """The old log-probabilities such that no ratio is within 1e-3 of where it is cut off (the gradients on the two sides differ)."""
    seen = {}

    class Look(_Plain):
        @classmethod
        def policy_loss(cls, z, t, *a, **k):
            seen["logp"] = cls.token_logprob(z, t, 0.3)
            return z.sum(), None
    _model(Look, tokens, targets, {k: v.double() for k, v in params.items()}, {})
    ahead = torch.linspace(-0.4, 0.4, ROWS, device="cuda").double()
    for edge in (0.8, 1.2):
        ahead = torch.where((ahead.exp() - edge).abs() < 1e-3, ahead + 5e-3, ahead)
    given["old_logp"] = (seen["logp"] - ahead).float()
    return given


def _grads(L, dtype, seed=0):
    tokens, targets, params, given = _inputs(seed)
    given = _off_the_edges(given, tokens, targets, params)
    p = {k: v.to(dtype).requires_grad_() for k, v in params.items()}
    loss = _model(L, tokens, targets, p, {k: v.to(dtype) for k, v in given.items()})
    return loss.detach(), torch.autograd.grad(loss, list(p.values()))


def test_together_against_64_bits(layers):
    """fp32 throughout.  Every operator is right to some 2^-24 of its terms' magnitudes and so is the product for the logits; sums of 50 rows and of 300 columns of terms of either sign
    leave 64 times that, of the largest entry."""
    loss, grads = _grads(layers, torch.float32)
    ref, refs = _grads(_Plain, torch.float64)
    assert abs(float(loss) - float(ref)) <= 64 * 2.0 ** -24 * (1 + abs(float(ref)))
    for g, r in zip(grads, refs):
        assert float((g.double() - r).abs().max()) <= 64 * 2.0 ** -24 * float(r.abs().max())


@pytest.mark.parametrize("near", [False, True])
def test_together_against_differences(layers, near):
    """The loss of fp32 is off by some 2^-24 |loss|, so a difference of two over 2 h is off by that over h, and by h^2 times a third derivative of the loss's order.  (Where the reference
    is far from the policy, the loss is some 10^6: exp(f) of an f of 15 and more.)"""
    tokens, targets, params, given = _inputs(1)
    given = _off_the_edges(given, tokens, targets, params)
    if near:
        given["ref_logp"] = given["old_logp"] + 0.5
    p = {k: v.requires_grad_() for k, v in params.items()}
    grads = torch.autograd.grad(_model(layers, tokens, targets, p, given), list(p.values()))
    g = torch.Generator().manual_seed(9)
    for (name, t), grad in zip(p.items(), grads):
        d = torch.randn(t.shape, generator=g).cuda()
        d /= d.norm()
        h = 4e-3
        with torch.no_grad():
            up, down = (float(_model(layers, tokens, targets, {**p, name: t + s * d}, given)) for s in (h, -h))
        assert abs((up - down) / (2 * h) - float((grad * d).sum())) <= (64 * 2.0 ** -24 / h + 10 * h * h) * (1 + abs(up)), name


def test_gradients_of_either_form_are_the_same(layers):
    """In one pass with the loss, or from the logits once more: the same numbers to the rounding of lse."""
    from paper_2601_22137_amd import prism
    tokens, targets, params, given = _inputs(2)
    z = (3 * torch.randn(ROWS, V, device="cuda")).requires_grad_()
    loss, logp = layers.policy_loss(z, targets, kl=0.1, **given)
    (2 * loss).backward()
    r = prism.policy_loss(z.detach(), targets, kl=0.1, **given)
    assert torch.allclose(loss, r.loss, rtol=1e-6) and torch.allclose(logp, r.logp, rtol=1e-6)
    assert float((z.grad - 2 * r.dlogits).abs().max()) <= 64 * 2.0 ** -24 * float(z.grad.abs().max())


def test_bf16_and_modules(layers):
    torch.manual_seed(0)
    e, n = layers.Embedding(V, W), layers.LayerNorm(W)
    tokens, targets, _, _ = _inputs(3)
    x = e(tokens)
    y, total = n(x, residual=x)
    assert x.dtype is torch.bfloat16 and y.dtype is torch.bfloat16 and torch.equal(total, (x.float() * 2).bfloat16())
    loss, _ = layers.policy_loss(y @ e.weight.t(), targets)
    loss.backward()
    assert e.weight.grad.dtype is torch.bfloat16 and n.weight.grad.dtype is torch.float32
    assert all(bool(p.grad.isfinite().all()) and bool(p.grad.any()) for m in (e, n) for p in m.parameters())


def test_a_training_step_in_a_graph(layers):
    """Forward and backward captured, replayed on new tokens with eager steps between."""
    tokens, targets, params, given = _inputs(4)
    p = {k: v.requires_grad_() for k, v in params.items()}
    step = lambda: (lambda l: (l.detach(), *torch.autograd.grad(l, list(p.values()))))(_model(layers, tokens, targets, p, given))   # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step()
    g = torch.Generator().manual_seed(5)
    for _ in range(4):
        tokens.copy_(torch.randint(-1, V, (ROWS,), generator=g))
        targets.copy_(torch.randint(-1, V, (ROWS,), generator=g))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        # (the products of the logits may be added up in another order)
        for a, b in zip(out, want):
            assert float((a - b).abs().max()) <= 64 * 2.0 ** -24 * float(b.abs().max())


def test_example_policy_steps(layers):
    spec = importlib.util.spec_from_file_location("muon_attention", os.path.join(ROOT, "examples", "muon_attention.py"))
    M = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(M)
    torch.manual_seed(0)
    rewards, norms = M.tune(M.Model(), 2, answers=6, length=9, say=None)
    assert len(rewards) == 2 and len(norms) == 4 and all(0 <= r <= 1 for r in rewards) and all(n > 0 and n < float("inf") for n in norms)
