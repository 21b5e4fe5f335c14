"""The operators under autograd, the attention layer made of them, and the example that trains it: gradients against PyTorch's in 64 bits, token by token
against the whole sequence."""
import importlib.util
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def layers():
    from paper_2601_22137_amd import layers as M, prism
    prism.lib()
    return M


def _reference(x, m, positions, doc):
    """The layer in 64 bits, elementary operations only, without dropout."""
    b, n, _ = x.shape
    hq, hk, d = m.heads, m.k_heads, m.dim
    w = {k: v.detach().double().requires_grad_() for k, v in (("w_qkv", m.w_qkv), ("w_out", m.w_out), ("q_weight", m.q_weight), ("k_weight", m.k_weight))}
    q, k, v = (x @ w["w_qkv"].t()).view(b, n, hq + 2 * hk, d).split([hq, hk, hk], 2)
    angle = positions.double()[:, :, None, None] * m.inv_freq.double()
    cos, sin = angle.cos(), angle.sin()

    def turn(t, weight):
        t = t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6) * weight
        a, c = t[..., :d // 2], t[..., d // 2:]
        return torch.cat([a * cos - c * sin, c * cos + a * sin], -1)
    q, k = turn(q, w["q_weight"]), turn(k, w["k_weight"])
    k, v = (t.repeat_interleave(hq // hk, 2) for t in (k, v))
    s = torch.matmul(q.transpose(1, 2), k.permute(0, 2, 3, 1).contiguous()) * d ** -0.5
    if m.softcap:
        s = m.softcap * torch.tanh(s / m.softcap)
    i = torch.arange(n, device=x.device)
    see = (i[None, :] <= i[:, None]) & (doc[:, :, None] == doc[:, None, :]) & (doc[:, :, None] >= 0)
    p = torch.softmax(s.masked_fill(~see[:, None], -1e30), -1).masked_fill(~see[:, None], 0.0)
    y = torch.matmul(p, v.transpose(1, 2).contiguous()).transpose(1, 2).reshape(b, n, hq * d)
    return x + y @ w["w_out"].t(), w


@pytest.mark.parametrize("softcap,k_heads", [(0.0, 4), (5.0, 2)])
def test_layer_and_gradients(layers, softcap, k_heads):
    torch.manual_seed(3)
    m = layers.SelfAttention(96, 4, k_heads, head_dim=32, softcap=softcap, dtype=torch.float32)
    m.eval()
    with torch.no_grad():
        m.q_weight.mul_(1.5)
    x = torch.randn(2, 75, 96, device="cuda", requires_grad=True)
    doc = torch.tensor([[0] * 30 + [1] * 40 + [-1] * 5, [2] * 75], dtype=torch.int32, device="cuda")
    positions = torch.cat([torch.arange(30), torch.arange(45), torch.arange(75)]).int().view(2, 75).cuda()
    g = torch.randn(2, 75, 96, device="cuda")
    m(x, positions, doc).backward(g)
    x64 = x.detach().double().requires_grad_()
    y64, w = _reference(x64, m, positions, doc)
    y64.backward(g.double())
    # fp32 throughout: some hundred roundings of 2^-24 in every entry, which grow with the root of their number in the norms compared: 1e-5 is ten times that
    pairs = [(x.grad, x64.grad)] + [(getattr(m, k).grad, v.grad) for k, v in w.items()]
    for a, e in pairs:
        assert float((a.double() - e).norm() / e.norm()) < 1e-5


def test_dropout_gradient_is_the_mask(layers):
    x = torch.randn(1000, device="cuda", requires_grad=True)
    r = torch.randn(1000, device="cuda", requires_grad=True)
    y = layers.dropout(x, 0.25, 11, 3, residual=r)
    y.backward(torch.ones_like(y))
    kept = x.grad != 0
    assert torch.equal(x.grad[kept], torch.full_like(x.grad[kept], 65536 / 49152)) and torch.all(r.grad == 1)
    assert torch.allclose(y - r, torch.where(kept, x * (65536 / 49152), 0.0), atol=1e-6)


def test_token_by_token_is_the_sequence(layers):
    torch.manual_seed(4)
    m = layers.SelfAttention(64, 4, 2, head_dim=32, softcap=20.0, dtype=torch.float32)
    m.eval()
    x = torch.randn(3, 40, 64, device="cuda")
    with torch.no_grad():
        whole = m(x)
        cache = m.new_cache(3, 48)
        steps = torch.cat([m.step(x[:, i:i + 1], cache) for i in range(40)], 1)
    assert float((whole - steps).norm() / whole.norm()) < 2e-6
    assert cache[2].tolist() == [40] * 3


def test_gradients_of_expanded_and_unused(layers):
    """A gradient that autograd expands from one number, keys that are broadcast over the batch, a result that nothing reads."""
    q = torch.randn(2, 5, 2, 32, device="cuda", requires_grad=True)
    k = torch.randn(1, 7, 2, 32, device="cuda", requires_grad=True)
    out = layers.attention(q, k.expand(2, 7, 2, 32), k.expand(2, 7, 2, 32))
    out.sum().backward()
    q64, k64 = q.detach().double().requires_grad_(), k.detach().double().requires_grad_()
    s = torch.matmul(q64.transpose(1, 2), k64.permute(0, 2, 3, 1).contiguous()) * 32 ** -0.5
    torch.matmul(torch.softmax(s, -1), k64.transpose(1, 2).contiguous()).sum().backward()
    assert torch.allclose(k.grad.double(), k64.grad, atol=1e-5) and torch.allclose(q.grad.double(), q64.grad, atol=1e-5)
    a = torch.randn(1, 3, 2, 32, device="cuda", requires_grad=True)
    f = torch.ones(16, device="cuda")
    layers.norm_rope(a, a.detach(), inv_freq=f)[0].sum().backward()
    assert torch.isfinite(a.grad).all()


def test_example_learns(layers):
    spec = importlib.util.spec_from_file_location("muon_attention", os.path.join(ROOT, "examples", "muon_attention.py"))
    M = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(M)
    model, losses = M.train(40, say=None)
    assert np.all(np.isfinite(losses)) and np.mean(losses[-5:]) < 0.8 * losses[0]
    prompts = torch.randint(0, M.VOCABULARY, (3, 12), device="cuda")
    assert M.generate(model, prompts, 4).shape == (3, 16)


def test_norm_rope_of_queries_or_keys_alone(layers):
    q, k = (torch.randn(2, 9, h, 64, device="cuda", requires_grad=True) for h in (4, 2))
    w = torch.ones(64, device="cuda", requires_grad=True)
    f = torch.rand(16, device="cuda")
    g = [torch.randn_like(t) for t in (q, k)]
    torch.autograd.backward(layers.norm_rope(q, k, w, w, inv_freq=f), g)
    both = [t.grad for t in (q, k, w)]
    q.grad = k.grad = w.grad = None
    layers.norm_rope(q, None, w, inv_freq=f)[0].backward(g[0])
    layers.norm_rope(None, k, None, w, inv_freq=f)[1].backward(g[1])
    assert torch.equal(q.grad, both[0]) and torch.equal(k.grad, both[1])
    # sums of 108 terms in fp32, of a gradient turned (1.5 of its largest entry) times an entry of a normed head (8 at most)
    assert torch.allclose(w.grad, both[2], rtol=0, atol=2.0 ** -23 * 108 * 1.5 * 8 * max(float(x.abs().max()) for x in g))


def test_second_derivatives(layers):
    """Those of dropout are right, those of the others an error."""
    x, r = (torch.randn(1000, device="cuda", requires_grad=True) for _ in range(2))
    y = layers.dropout(x, 0.25, 11, 3, residual=r)
    (gx,) = torch.autograd.grad((y ** 2).sum(), x, create_graph=True)
    gx.sum().backward()
    kept = (layers.dropout(torch.ones_like(x), 0.25, 11, 3) != 0).float() * (65536 / 49152)
    assert torch.allclose(x.grad, 2 * kept * kept) and torch.allclose(r.grad, 2 * kept)
    q = torch.randn(1, 5, 2, 32, device="cuda", requires_grad=True)
    for call in (lambda: layers.attention(q, q, q), lambda: layers.norm_rope(q, q)[0]):
        (g,) = torch.autograd.grad((call() ** 2).sum(), q, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            g.sum().backward()


def test_step_in_a_graph(layers):
    """Captured after the lengths were set by hand, replayed on new tokens with eager work between; the same tokens eagerly; then past the cache's end, which only loses tokens."""
    torch.manual_seed(6)
    m = layers.SelfAttention(64, 4, 2, head_dim=32, dtype=torch.float32)
    m.eval()
    tokens = torch.randn(7, 3, 1, 64, device="cuda")
    x, cache, eager = tokens[0].clone(), m.new_cache(3, 5), m.new_cache(3, 5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.no_grad():
        m.step(x, cache)
        cache[2].zero_()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y = m.step(x, cache)
    for i in range(7):
        x.copy_(tokens[i])
        graph.replay()
        torch.cuda.synchronize()
        if i < 5:
            assert torch.equal(y, m.step(tokens[i], eager)) and torch.equal(cache[0], eager[0])
        assert torch.isfinite(y).all()
    for c in (cache, eager):
        from paper_2601_22137_amd import prism
        with pytest.raises(prism.PrismError, match="5 tokens"):
            m.step(x, c)
