"""Operators at the ends of a model where their numbers are hardest: tokens next to certain, logits that are no numbers, large logarithms of sums, a ratio on its border; and the
kernels that only long odd rows, rows at odd entries or large arrays of fp32 reach.

E = 2^-24 is the relative error of a rounding to fp32, U that of one to the type of the arrays."""
import numpy as np
import pytest
import torch

from oracle import ends_ref as R

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
E = 2.0 ** -24
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def prism():
    from paper_2601_22137_amd import prism as P
    P.lib()
    return P


def _u(dtype):
    return 2.0 ** -8 if dtype == BF16 else 2.0 ** -24


def _f64(t):
    return t.detach().cpu().double().numpy()


def _within(got, ref, bound, what):
    got = _f64(got)
    assert got.shape == ref.shape and np.all(np.isfinite(got)), what
    off = np.abs(got - ref) / np.maximum(bound, 1e-300)
    assert off.max(initial=0.0) <= 1.0, (what, float(off.max()), np.unravel_index(off.argmax(), off.shape))


# ------------------------------------------------------------------------------------------------- tokens next to certain

def _likely(rows, v, dtype, scale):
    """Rows whose token is 8 to 24 nats above the sum of the others; the first token, the last, one next to the last whole vector, some in the middle."""
    g = torch.Generator().manual_seed(rows + v)
    z = (2.0 * torch.randn(rows, v, generator=g)).to(dtype).double()
    t = torch.randint(0, v, (rows,), generator=g)
    t[0], t[1], t[2] = 0, v - 1, max(v - 9, 0)
    at = torch.arange(rows)
    z[at, t] = -INF
    z[at, t] = (torch.logsumexp(scale * z, 1) + torch.linspace(8.0, 24.0, rows, dtype=torch.float64)) / scale
    return z.to(dtype).cuda(), t.cuda()


def _off_others(z, tokens, scale, v):
    """(what the sum of a row's other exponentials may be off by, relative; the distances of the logits from the others' largest; that).

    An exponential is off by its exponent's roundings (difference, factor, product: 3 E of it) and the instruction's, 3 E.  A thread adds up to v / 64 or v / (4 * 512) of them in vectors of
    four, 8 E each with what it raises its reference by; 16 joins of 5 E."""
    a = scale * z
    a[np.arange(len(a)), tokens] = -INF
    top = a.max(1, keepdims=True)
    far = np.where(np.isfinite(a), top - np.where(np.isfinite(a), a, 0.0), 0.0)
    w = np.where(np.isfinite(a), np.exp(-far), 0.0)
    vectors = max(v / (64 * 4) if v <= 8192 else v / (256 * 4) if v <= 32768 else v / (512 * 4), 1.0)
    return E * (3 * (w * far).sum(1) / w.sum(1) + 8 * (vectors + 1) + 83), far, top[:, 0]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [1.0, 0.7])
@pytest.mark.parametrize("rows,v", [(12, 2), (40, 64), (23, 1000), (9, 5000), (8, 32768), (7, 50001), (5, 131080)])
def test_tokens_next_to_certain(prism, dtype, scale, rows, v):
    """logp, 1 - p and the token's gradient keep their relative precision, whatever is left of 1: they follow from the sum of the others."""
    z, t = _likely(rows, v, dtype, scale)
    at, tokens = np.arange(rows), t.cpu().numpy()
    logp_ref, rest, p = R.logprob_apart(_f64(z), tokens.tolist(), scale)
    off, far, top = _off_others(_f64(z), tokens, scale, v)
    # the sum, the token's exponential beside it (3 E), the result
    off_logp = (off + 5 * E) * np.abs(logp_ref)
    lse_ref = scale * _f64(z)[at, tokens] - logp_ref
    logp, lse = prism.token_logprob(z, t, scale=scale)
    _within(logp, logp_ref, off_logp, "logp")
    assert bool((logp < 0).all())
    _within(lse, lse_ref, off_logp + E * np.abs(lse_ref), "lse")

    def gradient(d):
        g = R.logprob_gradient(d, p, tokens.tolist(), scale)
        g[at, tokens] = scale * d * rest
        return g
    # in one pass with the loss: 3 E of an exponent; the sum, and 1 - p, which is in error by the sum's error; ten roundings of factors and the result's
    d = torch.linspace(0.5, 1.5, rows).cuda()
    r = prism.policy_loss(z, t, weights=d, scale=scale)
    ref = gradient(-_f64(d))
    relative = 3 * E * far + (2 * off + 10 * E)[:, None] + _u(dtype)
    relative[at, tokens] = off + 10 * E + _u(dtype)
    _within(r.logp, logp_ref, off_logp, "logp of the loss")
    _within(r.loss.view(1), np.array([-(_f64(d) * logp_ref).sum()]), (_f64(d) * off_logp).sum() + E * (_f64(d) * np.abs(logp_ref)).sum(), "loss")
    _within(r.dlogits, ref, relative * np.abs(ref) + 1e-37, "dlogits of the loss")
    # from lse, which is rounded: all of a row by the same factor; distances from it rather than from the others' largest.  The token's is the others' share, added up like their sum and without that factor.
    ref = gradient(_f64(d))
    further = 3 * E * np.abs(lse_ref - top)
    relative = 3 * E * far + (2 * off + further + E * np.abs(lse_ref) + 10 * E)[:, None] + _u(dtype)
    relative[at, tokens] = off + further + 10 * E + _u(dtype)
    _within(prism.token_logprob_backward(d, z, t, lse, scale=scale), ref, relative * np.abs(ref) + 1e-37, "dlogits")
    place = z.clone()
    assert torch.equal(prism.token_logprob_backward(d, z, t, lse, scale=scale), prism.token_logprob_backward(d, place, t, lse, scale=scale, out=place))


# --------------------------------------------------------------------------------------------------- what is no number

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("v", [2, 40, 5000, 65544, 131080])
def test_rows_with_logits_that_are_no_numbers(prism, dtype, v):
    """A NaN or +inf among a row's logits is NaN in all that the row has, its whole gradient among it, and in no other row."""
    g = torch.Generator().manual_seed(v)
    z, t = torch.randn(8, v, generator=g).to(dtype).cuda(), torch.randint(0, v, (8,), generator=g)
    clean = z.clone()
    other = (t + 1) % v
    z[1, other[1]], z[2, other[2]], z[3, t[3]], z[4, t[4]] = NAN, INF, NAN, INF
    z[6] = -INF
    z[6, t[6]] = NAN
    t[7], z[7] = -1, NAN
    t, bad, good = t.cuda(), [1, 2, 3, 4, 6], [0, 5]
    logp, lse = prism.token_logprob(z, t)
    want = prism.token_logprob(clean, t)
    d = prism.token_logprob_backward(torch.ones(8, device="cuda"), z, t, lse)
    assert bool(logp[bad].isnan().all()) and bool(lse[bad].isnan().all()) and bool(d[bad].isnan().all())
    assert torch.equal(logp[good], want[0][good]) and torch.equal(lse[good], want[1][good]) and logp[7] == 0 and lse[7] == 0
    assert torch.equal(d[good], prism.token_logprob_backward(torch.ones(8, device="cuda"), clean, t, lse)[good]) and not bool(d[7].any())
    given = dict(advantages=torch.linspace(-1, 1, 8).cuda(), old_logp=want[0] - 0.1, ref_logp=want[0] + 0.1, kl=0.1)
    for kw in ({}, given, dict(given, kl=0.0)):
        r, c = prism.policy_loss(z, t, **kw), prism.policy_loss(clean, t, **kw)
        assert bool(r.loss.isnan()) and bool(r.dlogits[bad].isnan().all()) and torch.equal(r.dlogits[good], c.dlogits[good]) and not bool(r.dlogits[7].any())
        assert bool(r.dlogp[bad].isnan().all()) if kw else torch.equal(r.dlogp, c.dlogp)         # without a ratio it does not depend on logp
        assert torch.equal(r.dlogp[good], c.dlogp[good]) and bool(r.logp[bad].isnan().all())


def test_ratios_that_are_no_numbers(prism):
    """An advantage or an old log-probability that is no number is one in the gradient; an infinite ratio without an advantage adds nothing."""
    z, t = torch.randn(4, 30, device="cuda"), torch.arange(4, device="cuda")
    logp, _ = prism.token_logprob(z, t)
    old, a = logp.clone(), torch.ones(4, device="cuda")
    old[1], a[2], old[3], a[3] = NAN, NAN, -INF, 0.0
    r = prism.policy_loss(z, t, advantages=a, old_logp=old, weights=torch.ones(4, device="cuda"))
    assert r.dlogp.isnan().tolist() == [False, True, True, False] and r.dlogits.isnan().all(1).tolist() == [False, True, True, False]
    assert r.dlogp[3] == 0 and not bool(r.dlogits[3].any())
    r = prism.policy_loss(z[3:], t[3:], advantages=a[3:], old_logp=old[3:])
    assert r.loss == 0


# ------------------------------------------------------------------------------------------------ large logarithms of sums

@pytest.mark.parametrize("v", [3, 300, 5000, 40000, 65541])
def test_probabilities_of_rows_with_a_large_lse(prism, v):
    """fp32: lse is rounded by up to 2^-24 |lse|, 32 E here, which the probabilities do not take over.  Three logits close together, the others excluded: an exponent's roundings are 3 E of 0.25, in the probability and
    in the sum; two sums, two instructions of 2 E, the reciprocal's 2 E and six roundings of products each side."""
    g = torch.Generator().manual_seed(3)
    rows = 500
    z = torch.empty(rows, 3).uniform_(40.0, 62.0, generator=g)[:, :1] + 0.25 * torch.rand(rows, 3, generator=g)
    z[::2] -= 100.0
    t = torch.randint(0, 3, (rows,), generator=g)
    places = torch.arange(3) * (v - 1) // 2
    z, t = torch.full((rows, v), -INF, device="cuda").index_copy_(1, places.cuda(), z.cuda()), places[t].cuda()
    _, lse = prism.token_logprob(z, t)
    _, rest, p = R.logprob_apart(_f64(z), t.tolist(), 1.0)
    d = torch.rand(rows, generator=g).cuda()
    ref = R.logprob_gradient(_f64(d), p, t.tolist(), 1.0)
    ref[np.arange(rows), t.cpu().numpy()] = _f64(d) * rest
    _within(prism.token_logprob_backward(d, z, t, lse), ref, (2 * 3 * 0.25 + 2 + 4 + 2 + 12) * E * np.abs(ref), "dlogits")


# --------------------------------------------------------------------------------------------------- a ratio on its border

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("v", [1, 300, 5000, 140000])
def test_a_ratio_on_its_border_has_the_gradient_of_the_ratio(prism, dtype, v):
    """Tokens without another logit: logp is 0, the ratio 1 and nothing is lost to rounding; held between 1 and 1.  And where there are others the gradient reaches them."""
    z = torch.full((4, v), -INF, dtype=dtype, device="cuda")
    t = torch.tensor([0, v // 2, v - 1, 0], device="cuda")
    z[torch.arange(4), t] = torch.tensor([0.0, 3.0, -7.0, 1.5], dtype=dtype, device="cuda")
    a, w = torch.tensor([1.0, -1.0, 2.0, -0.5], device="cuda"), torch.ones(4, device="cuda")
    r = prism.policy_loss(z, t, advantages=a, old_logp=torch.zeros(4, device="cuda"), weights=w, clip=(0.0, 0.0))
    assert torch.equal(r.logp, torch.zeros(4, device="cuda")) and torch.equal(r.dlogp, -a) and r.loss == -a.sum() and not bool(r.dlogits.any())
    if v > 1:
        z[torch.arange(4), (t + 1) % v] = z[torch.arange(4), t]
        logp, _ = prism.token_logprob(z, t)                  # -log 2, rounded: the ratio is off by 2^-24 at most
        r = prism.policy_loss(z, t, advantages=a, old_logp=logp, weights=w, clip=(0.25, 0.25))
        assert bool(((r.dlogp + a).abs() <= 4 * E * a.abs()).all()) and bool(((r.dlogits[torch.arange(4), t].float() + a / 2).abs() <= (_u(dtype) + 8 * E) * a.abs()).all())


# ------------------------------------------------------------------------- rows of the norm at odd entries, and long odd ones

def _at_odd_entries(t):
    whole = torch.full((t.shape[0], t.shape[1] + 5), NAN, dtype=t.dtype, device="cuda")
    whole[:, 3:3 + t.shape[1]] = t
    view = whole[:, 3:3 + t.shape[1]]
    assert not view.is_contiguous() or t.shape[0] == 1
    return view


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,width", [(1, 1), (3, 2), (5, 8), (257, 64), (70, 100), (11, 129), (9, 513), (20, 768), (2, 1111), (3, 2050), (3, 4096), (2, 5001), (2, 7001), (2, 8200), (2, 16383)])
def test_norm_of_rows_at_odd_entries(prism, dtype, rows, width):
    """The same bits as those of rows next to each other, with NaN around each row."""
    g = torch.Generator(device="cuda").manual_seed(rows + width)
    make = lambda: torch.randn(rows, width, generator=g, device="cuda").to(dtype)   # noqa: E731
    x, r, dy, dt, w = make(), make(), make(), make(), torch.rand(width, generator=g, device="cuda")
    for res in (None, r):
        y, total, stats = prism.layer_norm(x, w, residual=res)
        got = prism.layer_norm(_at_odd_entries(x), w, residual=None if res is None else _at_odd_entries(res))
        assert torch.equal(got[0], y) and torch.equal(got[1], total) and torch.equal(got[2], stats)
        want = prism.layer_norm_backward(dy, total, stats, w, dtotal=None if res is None else dt)
        got = prism.layer_norm_backward(_at_odd_entries(dy), _at_odd_entries(total), stats, w, dtotal=None if res is None else _at_odd_entries(dt))
        assert all(torch.equal(a, b) for a, b in zip(got, want))


# 1024 threads a row with part of a vector at its end: over 3 * 256 vectors
@pytest.mark.parametrize("dtype,width", [(F32, 3079), (F32, 8193), (F32, 16383), (BF16, 6147), (BF16, 9001), (BF16, 16383)])
@pytest.mark.parametrize("center,residual,affine", [(True, False, True), (True, True, True), (False, True, True), (False, False, False)])
@pytest.mark.parametrize("rows", [2, 600])
def test_norm_of_long_odd_rows(prism, dtype, width, center, residual, affine, rows):
    """Against the oracle, with the bounds of the other widths."""
    import test_gpu_ends
    test_gpu_ends.test_layer_norm_and_gradients(prism, dtype, center, residual, affine, "plain" if rows > 2 else "odd", rows, width)


# ------------------------------------------------------------------------------------------- large arrays of fp32

def _parts(rows, size):
    return [slice(a, a + size) for a in (0, rows // 2, rows - size)]


@pytest.mark.parametrize("dtype,v", [(F32, 200), (F32, 2000), (F32, 4000), (F32, 8000), (F32, 16384), (F32, 32768), (F32, 65536), (F32, 66001), (BF16, 2000), (BF16, 4000), (BF16, 8000), (BF16, 16384)])
def test_logits_larger_than_the_caches(prism, dtype, v):
    """Kernels that read past the caches, of every number of threads: rows are the same bits as in calls of a part of them."""
    g = torch.Generator(device="cuda").manual_seed(v)
    rows = (300 << 20) // (v * (4 if dtype == F32 else 2))
    z, t = torch.randn(rows, v, generator=g, device="cuda").to(dtype), torch.randint(-1, v, (rows,), generator=g, device="cuda")
    w, old = torch.rand(rows, generator=g, device="cuda"), torch.full((rows,), -12.0, device="cuda")
    logp, lse = prism.token_logprob(z, t)
    r = prism.policy_loss(z, t, old_logp=old, weights=w)
    for part in _parts(rows, 70):
        b = prism.policy_loss(z[part], t[part], old_logp=old[part], weights=w[part])
        assert torch.equal(r.dlogits[part], b.dlogits) and torch.equal(r.logp[part], b.logp)
        c = prism.token_logprob(z[part], t[part])
        assert torch.equal(logp[part], c[0]) and torch.equal(lse[part], c[1])


@pytest.mark.parametrize("width", [100, 101, 768, 771, 4096, 4099, 8192, 16384, 16383])
def test_norm_of_fp32_larger_than_the_caches(prism, width):
    g = torch.Generator(device="cuda").manual_seed(width)
    rows = (100 << 20) // (4 * width)
    make = lambda: torch.randn(rows, width, generator=g, device="cuda")   # noqa: E731
    x, res, weight = make(), make(), torch.rand(width, generator=g, device="cuda")
    y, total, stats = prism.layer_norm(x, weight, residual=res)
    dx, dw, db = prism.layer_norm_backward(y, total, stats, weight, dtotal=res)
    for part in _parts(rows, 300):
        b = prism.layer_norm(x[part], weight, residual=res[part])
        assert all(torch.equal(p, q) for p, q in zip(b, (y[part], total[part], stats[part])))
        assert torch.equal(dx[part], prism.layer_norm_backward(y[part], total[part], stats[part], weight, dtotal=res[part])[0])
    n = (total.double() - stats[:, :1].double()) * stats[:, 1:].double()
    for got, terms in ((dw, y.double() * n), (db, y.double())):
        # 256 workgroups at least, and so rows / 256 terms a thread at most; n is off by two roundings, and parts are joined
        assert bool(((got.double() - terms.sum(0)).abs() <= (rows // 256 + 40) * E * terms.abs().sum(0)).all())


def test_gradient_of_log_probabilities_of_many_rows(prism):
    """More rows than one launch has workgroups for: from lse, or their sums once more, like those of a call of fewer, to the rounding of lse and some of each exponential."""
    rows = (1 << 20) + 300
    g = torch.Generator(device="cuda").manual_seed(1)
    z, t = torch.randn(rows, 5, generator=g, device="cuda"), torch.randint(-1, 5, (rows,), generator=g, device="cuda")
    z[::3] += 80.0
    z[1::7] -= 40.0
    z[torch.arange(rows, device="cuda"), t.clamp(min=0)] += 12.0 * torch.rand(rows, generator=g, device="cuda")
    d = torch.rand(rows, generator=g, device="cuda") + 0.5
    _, lse = prism.token_logprob(z, t)
    got = prism.token_logprob_backward(d, z, t, lse)
    half = rows // 2
    want = torch.cat([prism.token_logprob_backward(d[part], z[part], t[part], lse[part]) for part in (slice(0, half), slice(half, rows))])
    # exponents of 20 at most: 3 E of that on either side, 20 E of factors and sums, and 32 E of lse
    assert bool(((got - want).abs() <= (2 * 3 * 20 + 2 * 20 + 32) * E * want.abs()).all())
    assert not bool(got[t < 0].any())
    assert torch.equal(got, prism.token_logprob_backward(d, z, t, lse, out=z))


def test_embedding_of_fp32_larger_than_the_caches(prism):
    g = torch.Generator(device="cuda").manual_seed(1)
    n, rows, width = 40000, 12000, 1000
    dout, table, t = torch.randn(n, width, generator=g, device="cuda"), torch.randn(rows, width, generator=g, device="cuda"), torch.randint(-1, rows, (n,), generator=g, device="cuda")
    out = prism.embedding(t, table, scale=0.5)
    assert torch.equal(out, torch.where((t >= 0).unsqueeze(1), table[t.clamp(min=0)] * 0.5, torch.zeros((), device="cuda")))
    d = prism.embedding_backward(dout, t, rows)
    whole = torch.zeros(rows, width, device="cuda", dtype=torch.float64).index_add_(0, t.clamp(min=0), torch.where((t >= 0).unsqueeze(1), dout.double(), 0.0))
    size = torch.zeros(rows, width, device="cuda", dtype=torch.float64).index_add_(0, t.clamp(min=0), torch.where((t >= 0).unsqueeze(1), dout.abs().double(), 0.0))
    # 64 terms one after the other at most, parts rounded, joined in 64 bits, rounded
    assert bool(((d.double() - whole).abs() <= 67 * E * size).all())
