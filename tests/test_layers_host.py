"""What layers.py does around the library's calls, with stand-ins for them that need no GPU: only how gradients, masks and caches are handed on is tested here."""
import pytest
import torch

from paper_2601_22137_amd import layers, prism


@pytest.fixture(autouse=True)
def stand_ins(monkeypatch):
    """Calls of the right shapes; results keep a trace of what they were made from."""
    def qk_norm_rope(q, k, **kw):
        return tuple(None if t is None else 2 * t for t in (q, k))

    def qk_norm_rope_backward(dq_out, dk_out, q, k, q_weight=None, k_weight=None, **kw):
        assert (dq_out is None) == (q is None) and (dk_out is None) == (k is None)
        return tuple(None if t is None else 2 * t for t in (dq_out, dk_out)) + tuple(None if t is None else t.sum((0, 1, 2)) for t in (q, k))

    def attention(q, k, v, **kw):
        return q + v.mean(), torch.zeros(q.shape[0], q.shape[2], q.shape[1])

    def attention_backward(dout, q, k, v, out, lse, **kw):
        return dout.clone(), torch.zeros_like(k), torch.full_like(v, float(dout.sum()) / v.numel())

    def dropout(x, p, seed, offset=0, residual=None, out=None):
        y = x * float((seed + offset) % 7 + 1)
        return y if residual is None else y + residual
    for f in (qk_norm_rope, qk_norm_rope_backward, attention, attention_backward, dropout):
        monkeypatch.setattr(prism, f.__name__, torch.no_grad()(f))       # like the library, which autograd does not see into


def _heads(*shape):
    return torch.randn(*shape, requires_grad=True)


def test_norm_rope_of_queries_or_keys_alone():
    q, w = _heads(1, 3, 2, 8), torch.ones(8, requires_grad=True)
    a, none = layers.norm_rope(q, None, w)
    a.sum().backward()
    assert none is None and torch.all(q.grad == 2) and w.grad.shape == (8,)
    k = _heads(1, 3, 2, 8)
    none, b = layers.norm_rope(None, k)
    b.sum().backward()
    assert none is None and torch.all(k.grad == 2)


@pytest.mark.parametrize("call", [lambda q, k: layers.norm_rope(q, k)[0], lambda q, k: layers.attention(q, k, k)])
def test_second_derivatives_are_refused(call):
    """They are not computed; without an error a penalty on a gradient would quietly lose its part through these calls."""
    q, k = _heads(1, 3, 2, 8), _heads(1, 3, 2, 8)
    (g,) = torch.autograd.grad((call(q, k) ** 2).sum(), q, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (g ** 2).sum().backward()


def test_second_derivatives_of_dropout():
    x, r = _heads(5), _heads(5)
    y = layers.dropout(x, 0.5, 2, residual=r)        # the stand-in: 3 x + r
    gx, gr = torch.autograd.grad((y ** 3).sum(), (x, r), create_graph=True)
    (gx.sum() + gr.sum()).backward()
    z = (3 * x + r).detach()
    assert torch.allclose(x.grad, 3 * (3 + 1) * 6 * z) and torch.allclose(r.grad, (3 + 1) * 6 * z)


def test_results_have_no_given_place():
    """The backward pass would write its own results there."""
    q, k = _heads(1, 3, 2, 8), _heads(1, 3, 2, 8)
    with pytest.raises(TypeError, match="out"):
        layers.norm_rope(q, k, out=(torch.empty(1, 3, 2, 8), torch.empty(1, 3, 2, 8)))
    with pytest.raises(TypeError, match="out"):
        layers.attention(q, k, k, out=torch.empty(1, 3, 2, 8))
    with pytest.raises(TypeError):
        layers.attention(q, k, k, soft_cap=1.0)


@pytest.mark.parametrize("name", ["inv_freq", "positions", "q_weight"])
def test_norm_rope_notices_what_was_written_before_backward(name):
    q, k = _heads(1, 3, 2, 8), _heads(1, 3, 2, 8)
    given = dict(inv_freq=torch.ones(4), positions=torch.zeros(1, 3, dtype=torch.int32), q_weight=torch.ones(8))
    a, b = layers.norm_rope(q, k, **given)
    given[name].add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        (a.sum() + b.sum()).backward()


@pytest.mark.parametrize("name", ["slopes", "prefix", "k_lens", "q_doc", "k_doc"])
def test_attention_notices_what_was_written_before_backward(name):
    q, k = _heads(2, 3, 2, 8), _heads(2, 3, 2, 8)
    i32 = lambda *s: torch.ones(*s, dtype=torch.int32)   # noqa: E731
    given = dict(slopes=torch.ones(2), prefix=i32(2), k_lens=i32(2), q_doc=i32(2, 3), k_doc=i32(2, 3))
    y = layers.attention(q, k, k, causal=True, workspace=torch.empty(1), **given)
    given[name].add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_scratch_memory_is_no_input():
    q, ws = _heads(1, 3, 2, 8), torch.zeros(4)
    y = layers.attention(q, q, q, workspace=ws)
    ws.add_(1)
    y.sum().backward()
    assert q.grad is not None


def test_learned_slopes_and_frequencies_are_refused():
    q = _heads(1, 3, 2, 8)
    learned = torch.ones(2, requires_grad=True)
    with pytest.raises(prism.PrismError, match="slopes"):
        layers.attention(q, q, q, slopes=learned)
    with pytest.raises(prism.PrismError, match="inv_freq"):
        layers.norm_rope(q, q, inv_freq=learned)
    with torch.no_grad():
        layers.attention(q, q, q, slopes=learned)
        layers.norm_rope(q, q, inv_freq=learned)


def _layer():
    return layers.SelfAttention(16, 2, device="cpu", dtype=torch.float32)


def test_a_full_cache_is_refused():
    m, x = _layer(), torch.randn(3, 1, 16)
    cache = m.new_cache(3, 4)
    keys, values, lens = cache
    for i in range(4):
        assert lens.tolist() == [i] * 3
        m.step(x, cache)
    before = [t.clone() for t in cache]
    with pytest.raises(prism.PrismError, match="4 tokens"):
        m.step(x, cache)
    assert all(torch.equal(a, b) for a, b in zip(before, cache))
    lens.fill_(0)                         # emptied, or filled by hand
    m.step(x, cache)
    lens.copy_(torch.tensor([0, 4, 1]))
    with pytest.raises(prism.PrismError, match="4 tokens"):
        m.step(x, cache)
    with pytest.raises(prism.PrismError, match="4 tokens"):
        m.step(x, (keys, values, lens))   # a plain tuple of the three
    lens.copy_(torch.tensor([0, 3, 1]))
    m.step(x, (keys, values, lens))
    assert lens.tolist() == [1, 4, 2]


def test_a_cache_under_inference_mode():
    with torch.inference_mode():
        m, x = _layer(), torch.randn(3, 1, 16)
        cache = m.new_cache(3, 2)
        m.step(x, cache)
        m.step(x, cache)
        with pytest.raises(prism.PrismError, match="2 tokens"):
            m.step(x, cache)
        with pytest.raises(prism.PrismError, match="2 tokens"):
            m.step(x, tuple(cache))


def test_masks_of_dropout_differ_unless_asked_for(monkeypatch):
    """In training every layer and step has a mask of its own; a seed or an offset names one; PyTorch's generator repeats them."""
    seen = []

    @torch.no_grad()
    def dropout(x, p, seed, offset=0, residual=None, out=None):
        seen.append((p, seed, offset))
        return x + residual
    monkeypatch.setattr(prism, "dropout", dropout)
    x = torch.randn(1, 3, 16)
    two = [layers.SelfAttention(16, 2, p=0.5, device="cpu", dtype=torch.float32) for _ in range(2)]

    def run(*args, **kw):
        del seen[:]
        for _ in range(3):
            for m in two:
                m(x, *args, **kw)
        return list(seen)
    torch.manual_seed(5)
    first = run()
    assert len({s for _, s, _ in first}) == 6 and all(0 <= s < 2 ** 63 and o == 0 and p == 0.5 for p, s, o in first)
    torch.manual_seed(5)
    assert run() == first
    assert set(run(seed=7, offset=3)) == {(0.5, 7, 3)} and set(run(seed=7)) == {(0.5, 7, 0)} and set(run(offset=3)) == {(0.5, 0, 3)} and set(run(seed=0)) == {(0.5, 0, 0)}
    state = torch.get_rng_state()
    for m in two:
        m.eval()
    assert {p for p, _, _ in run()} == {0.0} and torch.equal(state, torch.get_rng_state())


def test_drawn_seeds_are_of_the_host():
    m, x = layers.SelfAttention(16, 2, p=0.5, device="cpu", dtype=torch.float32), torch.randn(1, 3, 16)
    with torch.device("meta"):            # as a program does whose default device is the GPU
        m(x)


def test_no_part_of_a_head_turns(monkeypatch):
    seen = []
    plain = prism.qk_norm_rope
    monkeypatch.setattr(prism, "qk_norm_rope", lambda q, k, **kw: (seen.append(kw["inv_freq"]), plain(q, k, **kw))[1])
    for rot, frequencies in ((0, 0), (4, 2), (None, 4)):
        m = layers.SelfAttention(16, 2, rot_dim=rot, device="cpu", dtype=torch.float32)
        m(torch.randn(1, 3, 16))
        assert (0 if seen[-1] is None else seen[-1].numel()) == frequencies


def test_caches_are_copied(tmp_path):
    import copy
    import pickle
    m, x = _layer(), torch.randn(2, 1, 16)
    cache = m.new_cache(2, 2)
    m.step(x, cache)
    for other in (copy.deepcopy(cache), pickle.loads(pickle.dumps(cache)), copy.copy(cache)):
        assert all(torch.equal(a, b) for a, b in zip(cache, other))
    other = copy.deepcopy(cache)
    m.step(x, other)
    assert cache[2].tolist() == [1, 1] and other[2].tolist() == [2, 2]
    with pytest.raises(prism.PrismError, match="2 tokens"):
        m.step(x, other)
    m.step(x, cache)


def test_a_step_that_is_captured_reads_nothing(monkeypatch):
    """While a stream is captured the lengths cannot be read; afterwards they change unseen, so they are read before every other step."""
    m, x = _layer(), torch.randn(2, 1, 16)
    cache = m.new_cache(2, 4)
    m.step(x, cache)
    cache[2].zero_()
    reads, capturing = [], [True]
    monkeypatch.setattr(layers, "_capturing", lambda t: capturing[0])
    monkeypatch.setattr(layers.Cache, "_read", lambda self, plain=layers.Cache._read: (reads.append(1), plain(self))[1])
    m.step(x, cache)
    assert not reads
    capturing[0] = False
    with torch.no_grad():
        cache[2].data.add_(2)             # replays, which no version tells of
    m.step(x, cache)
    assert len(reads) == 1 and cache[2].tolist() == [4, 4]
    with pytest.raises(prism.PrismError, match="4 tokens"):
        m.step(x, cache)
