"""The operators at the ends of a model (prism_embedding, prism_layer_norm, prism_token_logprob, prism_policy_loss and their gradients) through the C-ABI against the fp64
oracle.

Tolerances count roundings.  U is the relative error of one to the type of the arrays (bf16 2^-8, fp32 2^-24), E = 2^-24 that of fp32 arithmetic; a sum of terms of which a
thread adds k one after the other, and which threads join in a tree, is off by at most (k + the tree's height) E times the sum of their magnitudes."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import ends_ref as R

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
E = 2.0 ** -24


@pytest.fixture(scope="module")
def prism():
    from paper_2601_22137_amd import prism as P
    P.lib()
    return P


def _u(dtype):
    return 2.0 ** -8 if dtype == BF16 else 2.0 ** -24


def _f64(t):
    return t.detach().cpu().double().numpy()


def _close(got, ref, bound, what):
    got = _f64(got)
    assert got.shape == ref.shape, what
    assert np.all(np.isfinite(got) == np.isfinite(ref)), what
    same = np.isfinite(ref)
    assert np.array_equal(got[~same], ref[~same]), what
    off = np.abs(got[same] - ref[same]) - np.broadcast_to(bound, ref.shape)[same]
    assert off.size == 0 or off.max() <= 0, (what, float(off.max()), float(np.max(np.abs(got[same] - ref[same]))))


def _array(g, shape, dtype, scale=1.0, view="plain"):
    """Rows of random numbers: 'plain', or in a wider array that starts at an odd entry, whose other entries are NaN."""
    x = (scale * torch.randn(shape, generator=g)).to(dtype)
    if view == "plain":
        return x.cuda()
    whole = torch.full((shape[0], shape[1] + 5), float("nan"), dtype=dtype, device="cuda")
    whole[:, 3:3 + shape[1]] = x.cuda()
    return whole[:, 3:3 + shape[1]]


def _place(shape, dtype, view="plain"):
    """(where a result goes, a check that nothing around it was written to)."""
    if view == "plain":
        return torch.full(shape, float("nan"), dtype=dtype, device="cuda"), lambda: None
    whole = torch.full((shape[0] + 2, shape[1] + 5), 77.0, dtype=dtype, device="cuda")

    def untouched():
        rest = torch.ones_like(whole, dtype=torch.bool)
        rest[1:-1, 3:3 + shape[1]] = False
        assert bool((whole[rest] == 77.0).all())
    return whole[1:-1, 3:3 + shape[1]], untouched


# -------------------------------------------------------------------------------------------------------------- embedding

# tokens, rows of the table, width, which tokens
EMBEDDING = [(1, 1, 1, "any"), (1, 5, 8, "any"), (7, 3, 33, "any"), (64, 64, 64, "any"), (300, 10, 96, "any"), (5000, 1000, 40, "any"), (3000, 70001, 8, "any"),
             (70000, 50, 8, "any"), (2000, 600, 1111, "any"), (5000, 131072, 24, "hot"), (20000, 300, 16, "one"), (1000, 2000, 520, "hot"), (129, 7, 5, "none"), (600, 512, 48, "sorted"),
             (257, 513, 17, "last")]


def _tokens(g, n, rows, kind, dtype):
    t = torch.randint(-1, rows + 1, (n,), generator=g)          # padding on either side among them
    if kind == "hot":
        t[torch.rand(n, generator=g) < 0.6] = rows // 2
    elif kind == "one":
        t[:] = rows - 1
    elif kind == "none":
        t[:] = torch.where(torch.rand(n, generator=g) < 0.5, -(2 ** 31) if dtype is torch.int32 else -(2 ** 40), 2 ** 31 - 1 if dtype is torch.int32 else 2 ** 40)
    elif kind == "sorted":
        t = t.sort().values
    elif kind == "last":
        t = rows - 1 - (t.clamp(0, rows - 1) % 3)
    return t.to(dtype).cuda()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
@pytest.mark.parametrize("view", ["plain", "odd"])
@pytest.mark.parametrize("n,rows,width,kind", EMBEDDING)
def test_embedding_and_gradient(prism, dtype, index, view, n, rows, width, kind):
    g = torch.Generator().manual_seed(n + rows)
    tokens, table, dout = _tokens(g, n, rows, kind, index), _array(g, (rows, width), dtype, view=view), _array(g, (n, width), dtype, view=view)
    scale = float(np.float32(width ** 0.5))
    out, untouched = _place((n, width), dtype, view)
    assert prism.embedding(tokens, table, scale=scale, out=out) is out
    ref = R.embedding(tokens.tolist(), _f64(table), scale)
    _close(out, ref, (_u(dtype) + E) * np.abs(ref), "out")        # the product, the result
    untouched()
    d, untouched = _place((rows, width), dtype, view)
    prism.embedding_backward(dout, tokens, rows, scale=scale, out=d)
    ref, size, count = R.embedding_gradient(_f64(dout), tokens.tolist(), rows, scale)
    # 64 terms one after the other at most, parts rounded, joined in 64 bits, rounded; the product; the result
    _close(d, ref, _u(dtype) * np.abs(ref) + (64 + 3) * E * size, "dtable")
    assert not bool(d[torch.from_numpy(count == 0).cuda()].any())
    untouched()
    assert torch.equal(d, prism.embedding_backward(dout, tokens, rows, scale=scale))


def test_embedding_shapes_and_nothing(prism):
    table = torch.randn(9, 6, device="cuda")
    tokens = torch.randint(0, 9, (2, 3, 4), device="cuda")
    out = prism.embedding(tokens, table)
    assert torch.equal(out, table[tokens])
    d = prism.embedding_backward(out, tokens, 9)
    assert d.shape == (9, 6)
    assert prism.embedding(tokens[:, :0], table).shape == (2, 0, 4, 6)
    assert not bool(prism.embedding_backward(out[:, :0], tokens[:, :0], 9).any())
    assert not bool(prism.embedding(tokens, table[:0]).any()) and prism.embedding_backward(out, tokens, 0).shape == (0, 6)
    one = torch.tensor(3, device="cuda")
    assert torch.equal(prism.embedding(one, table), table[3])
    same = table[:1].expand(24, 6)             # gradients of a broadcast
    assert torch.equal(prism.embedding_backward(same, tokens.view(-1), 9), prism.embedding_backward(same.contiguous(), tokens.view(-1), 9))


def test_embedding_nan_in_padding(prism):
    """Rows of dout whose token is padding are not read; infinities of a row stay in its own."""
    tokens = torch.tensor([0, -1, 2, 2, 5], device="cuda")
    d = torch.ones(5, 40, device="cuda", dtype=BF16)
    d[1], d[4], d[3, 7] = float("nan"), float("nan"), float("inf")
    g = prism.embedding_backward(d, tokens, 5)
    ref = torch.zeros(5, 40, device="cuda", dtype=BF16)
    ref[0], ref[2] = 1, 2
    ref[2, 7] = float("inf")
    assert torch.equal(g, ref)


# ------------------------------------------------------------------------------------------------------------- layer norm

NORM = [(1, 1), (3, 2), (5, 8), (257, 64), (70, 100), (11, 129), (40, 333), (9, 513), (20, 768), (2, 1111), (5, 2048), (4, 2050), (3, 4096), (2, 5000), (2, 8192), (3, 8200), (2, 16384),
        (9000, 96), (5000, 768), (1500, 2100)]


def _norm_bounds(h, w, b, center, eps, dtype):
    """(y and the rows before weight and bias, with what each may be off by before the result's rounding)."""
    y, n, mean, r = R.layer_norm(h, w, b, center, eps)
    # a thread adds at most 32 terms, trees of at most 6 + 16 levels; the division; the rounded mean
    off_mean = 56 * E * np.abs(h).mean(1, keepdims=True) if center else 0.0
    # the squares' sum likewise, two roundings a term, the division, eps, the root, its inverse: relative; and what the mean's error adds to the variance
    off_r = 35 * E + 0.5 * (off_mean * r) ** 2
    off_n = r * off_mean + (off_r + 4 * E) * np.abs(n)
    return y, n, off_n


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("center,residual,affine", [(True, False, True), (True, True, True), (False, True, True), (False, False, False)])
@pytest.mark.parametrize("view", ["plain", "odd"])
@pytest.mark.parametrize("rows,width", NORM)
def test_layer_norm_and_gradients(prism, dtype, center, residual, affine, view, rows, width):
    g = torch.Generator().manual_seed(rows + width)
    x = _array(g, (rows, width), dtype, 2.0, view) + (0 if view != "plain" else 1.5)
    res = _array(g, (rows, width), dtype, 3.0, view) if residual else None
    weight, bias = (1 + 0.3 * torch.randn(width, generator=g)).cuda() if affine else None, torch.randn(width, generator=g).cuda() if affine and center else None
    eps = float(np.float32(1e-5))
    y, y_untouched = _place((rows, width), dtype, view)
    total, t_untouched = _place((rows, width), dtype, view) if residual else (None, lambda: None)
    y, total, stats = prism.layer_norm(x, weight, bias, residual=res, center=center, eps=eps, out=(y, total))
    y_untouched()
    t_untouched()
    assert torch.equal(total, x if res is None else (x.float() + res.float()).to(dtype))
    h, w, b = _f64(total), _f64(weight) if affine else np.ones(width), _f64(bias) if bias is not None else np.zeros(width)
    ref, n, off_n = _norm_bounds(h, w, b, center, eps, dtype)
    _close(y, ref, _u(dtype) * np.abs(ref) + off_n * np.abs(w) + 3 * E * (np.abs(n * w) + np.abs(b)), "y")
    # gradients
    dy, dt = _array(g, (rows, width), dtype, 1.0, view), _array(g, (rows, width), dtype, 1.0, view) if residual else None
    dx, untouched = _place((rows, width), dtype, view)
    got = prism.layer_norm_backward(dy, total, stats, weight, dtotal=dt, center=center, bias=bias is not None, out=dx)
    untouched()
    d = _f64(dy)
    rdx, rdw, rdb = R.layer_norm_gradient(d, h, w, center, eps)
    _, _, _, r = R.layer_norm(h, w, b, center, eps)
    gw = d * w
    mean = lambda a: np.abs(a).mean(1, keepdims=True)   # noqa: E731
    p, s = np.abs((gw * n).mean(1, keepdims=True)), np.abs(gw.mean(1, keepdims=True)) if center else 0.0
    off_p, off_s = (np.abs(gw) * off_n).mean(1, keepdims=True) + 58 * E * mean(gw * n), 57 * E * mean(gw) if center else 0.0
    off_dx = r * (4 * E * (np.abs(gw) + s + np.abs(n) * p) + off_s + p * off_n + np.abs(n) * off_p) + 40 * E * np.abs(rdx)
    ref = rdx + (_f64(dt) if residual else 0.0)
    _close(got[0], ref, _u(dtype) * np.abs(ref) + off_dx + 2 * E * np.abs(ref), "dx")
    # a thread adds the rows that come to it: of 1024 workgroups, one to 16 rows at a time
    each = rows // 1024 + 4
    _close(got[1], rdw, (np.abs(d) * off_n).sum(0) + (each + 4) * E * np.abs(d * n).sum(0) + E * np.abs(rdw), "dw")
    if bias is not None:
        _close(got[2], rdb, (each + 4) * E * np.abs(d).sum(0) + E * np.abs(rdb), "db")
    else:
        assert got[2] is None
    again = prism.layer_norm_backward(dy, total, stats, weight, dtotal=dt, center=center, bias=bias is not None)
    assert all((a is None and c is None) or torch.equal(a, c) for a, c in zip(got, again))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_layer_norm_in_place(prism, dtype):
    g = torch.Generator().manual_seed(5)
    for rows, width in ((37, 768), (5, 4100)):
        x, r, w = _array(g, (rows, width), dtype), _array(g, (rows, width), dtype), torch.rand(width, device="cuda")
        y, total, stats = prism.layer_norm(x, w, residual=r)
        a, b = x.clone(), r.clone()
        prism.layer_norm(a, w, residual=b, out=(a, b))
        assert torch.equal(a, y) and torch.equal(b, total)
        a, b = x.clone(), r.clone()
        prism.layer_norm(a, w, residual=b, out=(b, a))
        assert torch.equal(b, y) and torch.equal(a, total)
        dy, dt = _array(g, (rows, width), dtype), _array(g, (rows, width), dtype)
        dx = prism.layer_norm_backward(dy, total, stats, w, dtotal=dt)[0]
        for place in (0, 1):
            given = [dy.clone(), dt.clone()]
            assert torch.equal(dx, prism.layer_norm_backward(given[0], total, stats, w, dtotal=given[1], out=given[place])[0])


def test_layer_norm_edges(prism):
    x = torch.full((3, 70), 5.0, device="cuda")
    y, total, stats = prism.layer_norm(x)                      # rows of one value: no variance
    assert total is x and not bool(y.any()) and torch.allclose(stats, torch.tensor([5.0, 1e-5 ** -0.5], device="cuda"))
    y, _, _ = prism.layer_norm(x, eps=0.0)
    assert bool(y.isnan().all())                               # 0 over 0, as the formula
    y, total, stats = prism.layer_norm(x[:0])
    dx, dw, db = prism.layer_norm_backward(y, total, stats)
    assert dx.shape == (0, 70) and not bool(dw.any()) and not bool(db.any())
    big = 1e4 + torch.randn(4, 1000, device="cuda")            # a mean far above the spread
    y = prism.layer_norm(big)[0]
    _close(y, *(lambda y, n, off: (y, E * np.abs(y) + off + 3 * E * np.abs(n)))(*_norm_bounds(_f64(big), np.ones(1000), np.zeros(1000), True, float(np.float32(1e-5)), F32)), "far mean")
    x = torch.randn(6, 40, device="cuda")
    x[2, 3], x[4, 5] = float("inf"), float("nan")              # rows do not touch one another
    y = prism.layer_norm(x)[0]
    assert y[[0, 1, 3, 5]].isfinite().all() and y[4].isnan().all()
    b = torch.randn(2, 3, 40, device="cuda")
    assert prism.layer_norm(b)[0].shape == (2, 3, 40)


# ------------------------------------------------------------------------------------------------- log-probabilities, losses

LOGITS = [(1, 1), (3, 2), (5, 7), (40, 64), (300, 65), (17, 1000), (9, 4096), (7, 4100), (5, 5000), (12, 10007), (4, 16384), (3, 32768), (2, 50001), (2, 65544), (3, 131072), (2, 131080), (1, 262145)]


def _logits(g, rows, v, dtype, view, index, hidden=True):
    z = _array(g, (rows, v), dtype, 3.0, view)
    t = torch.randint(0, v, (rows,), generator=g)
    if v > 1:
        z[torch.arange(rows), t.cuda()] += 6.0 * torch.rand(rows, generator=g).to(dtype).cuda()
    if hidden and v > 4:                                       # excluded logits; rows of padding, which hold NaN
        cut = torch.rand(rows, v, generator=g) < 0.1
        cut[torch.arange(rows), t] = False
        z[cut.cuda()] = -float("inf")
        for row, token in ((1, -1), (rows - 2, v)):
            if 0 < row < rows - 1:
                t[row], z[row] = token, float("nan")
    return z, t.to(index).cuda()


def _logprob_bounds(z, tokens, scale, v):
    """(logp, lse, p, what logp may be off by, what the logarithm of p may be off by), before results are rounded.

    An exponential is off by its factor's rounding (of the whole argument), the fused product's and the instruction's: E (|a| + |a - top| + 3), a = scale z.  A thread adds
    up to v / 64 or v / (4 * 512) exponentials in vectors, and each time raises its reference: 8 E a vector at most; 16 joins of 5 E."""
    logp, lse, p = R.logprob(z, tokens, scale)
    there = np.array([0 <= t < v for t in tokens])
    a = scale * np.where(there[:, None], z, 0.0)
    fin = np.isfinite(a)
    top = np.max(np.where(fin, a, -np.inf), axis=1, keepdims=True, initial=0.0)
    spread = np.where(fin, np.abs(a) + np.abs(a - np.where(np.isfinite(top), top, 0.0)), 0.0)
    vectors = max(v / (64 * 4) if v <= 4096 else v / (256 * 4) if v <= 16384 else v / (512 * 4), 1.0)
    off_sum = E * ((p * spread).sum(1) + 8 * (vectors + 1) + 83)
    taken = np.array([abs(a[i, t]) if there[i] and np.isfinite(a[i, t]) else 0.0 for i, t in enumerate(tokens)])
    off = off_sum + 3 * E * taken
    return logp, lse, p, off, E * (spread + 4) + off_sum[:, None]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("view,index", [("plain", torch.int64), ("odd", torch.int32)])
@pytest.mark.parametrize("scale", [1.0, 0.37])
@pytest.mark.parametrize("rows,v", LOGITS)
def test_token_logprob_and_gradient(prism, dtype, view, index, scale, rows, v):
    g = torch.Generator().manual_seed(rows + v)
    z, tokens = _logits(g, rows, v, dtype, view, index)
    s = scale
    logp, lse = prism.token_logprob(z, tokens, scale=scale)
    rlogp, rlse, p, off, off_p = _logprob_bounds(_f64(z), tokens.tolist(), s, v)
    _close(logp, rlogp, off + E * np.abs(rlogp), "logp")
    _close(lse, rlse, off + E * np.abs(rlse), "lse")
    dlogp = torch.randn(rows, generator=g).cuda()
    d, untouched = _place((rows, v), dtype, view)
    prism.token_logprob_backward(dlogp, z, tokens, lse, scale=scale, out=d)
    untouched()
    dl = _f64(dlogp)
    ref = R.logprob_gradient(dl, p, tokens.tolist(), s)
    size = s * np.abs(dl)[:, None]
    # the probability (lse rounded too), the product with s d, at the token the difference
    bound = _u(dtype) * np.abs(ref) + size * p * (off_p + (off + E * np.abs(rlse))[:, None] + 4 * E) + 2 * E * size * (p + (ref > 0) * (dl > 0)[:, None] + (ref < 0) * (dl < 0)[:, None]) + 1e-36
    _close(d, ref, bound, "dlogits")
    place = z.clone() if view == "plain" else z
    assert torch.equal(d, prism.token_logprob_backward(dlogp, place, tokens, lse, scale=scale, out=place))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("view,index", [("plain", torch.int32), ("odd", torch.int64)])
@pytest.mark.parametrize("old,weights,kl,scale", [(False, False, 0.0, 1.0), (True, True, 0.0, 1.0), (True, False, 0.3, 0.8), (False, True, 0.1, 1.3)])
@pytest.mark.parametrize("rows,v", LOGITS)
def test_policy_loss(prism, dtype, view, index, old, weights, kl, scale, rows, v):
    g = torch.Generator().manual_seed(rows + v)
    z, tokens = _logits(g, rows, v, dtype, view, index)
    s = scale
    rlogp, rlse, p, off, off_p = _logprob_bounds(_f64(z), tokens.tolist(), s, v)
    there = np.array([0 <= t < v for t in tokens.tolist()])
    given, ref = {}, {}
    if old:
        ahead = 0.3 * np.random.default_rng(rows).normal(size=rows)
        for edge in (np.log(0.8), np.log(1.3)):                # where the ratio is cut off the gradient jumps: not within what logp may be off by
            ahead = np.where(np.abs(ahead - edge) < 1e-2, edge + 2e-2, ahead)
        ahead[::5] = 0.0
        given["old_logp"], given["advantages"] = torch.from_numpy(rlogp - ahead).float().cuda(), torch.randn(rows, generator=g).cuda()
        ref["old"], ref["advantages"] = _f64(given["old_logp"]), _f64(given["advantages"])
    if weights:
        given["weights"] = torch.rand(rows, generator=g).cuda()
        given["weights"][::4] = 0.0
        ref["weights"] = _f64(given["weights"])
    if kl:
        given["ref_logp"] = torch.from_numpy(rlogp).float().cuda() + 0.4 * torch.randn(rows, generator=g).cuda()
        ref["ref"] = _f64(given["ref_logp"])
    place, untouched = _place((rows, v), dtype, view)
    r = prism.policy_loss(z, tokens, clip=(0.2, 0.3), kl=kl, scale=scale, out=place, **given)
    untouched()
    l, dl, second = R.policy_rows(rlogp, there, low=0.2, high=0.3, kl=kl, **ref)
    off_d = second * off + 2 * E * np.abs(dl)
    _close(r.logp, rlogp, off + E * np.abs(rlogp), "logp")
    _close(r.lse, rlse, off + E * np.abs(rlse), "lse")
    _close(r.loss.view(1), np.array([l.sum()]), (np.abs(dl) * off + second * off ** 2).sum() + 1e-13 * np.abs(l).sum() + E * abs(l.sum()), "loss")
    _close(r.dlogp, dl, off_d, "dlogp")
    ref_z = R.logprob_gradient(dl, p, tokens.tolist(), s)
    size, extra = s * np.abs(dl)[:, None], s * off_d[:, None]
    one = np.zeros_like(p)
    one[there, np.array(tokens.tolist())[there]] = 1.0
    _close(r.dlogits, ref_z, _u(dtype) * (np.abs(ref_z) + extra) + size * p * (off_p + 4 * E) + (extra + 2 * E * size) * (one + p) + 1e-36, "dlogits")
    # the same through the parts; the same bits again; without the gradient; in place of the logits
    assert all(torch.equal(a, b) for a, b in zip(r, prism.policy_loss(z, tokens, clip=(0.2, 0.3), kl=kl, scale=scale, **given)))
    part = prism.policy_loss(z, tokens, clip=(0.2, 0.3), kl=kl, scale=scale, gradient=False, **given)
    assert part.dlogits is None
    # (a row on its own may be added up in another order than with the gradient)
    _close(part.loss.view(1), np.array([l.sum()]), (np.abs(dl) * off + second * off ** 2).sum() + 1e-13 * np.abs(l).sum() + E * abs(l.sum()), "loss alone")
    r2 = prism.policy_loss(z, tokens, clip=(0.2, 0.3), kl=kl, scale=scale, out=z, **given)
    assert r2.dlogits is z and torch.equal(z, r.dlogits)


def test_logits_edges(prism):
    inf = float("inf")
    z = torch.zeros(6, 50, device="cuda")
    z[1], z[2, 1:], z[3, 7], z[4], z[5] = -inf, -inf, -inf, 1e4, -1e4
    z[5, 3] = 1e4
    t = torch.tensor([0, 4, 0, 7, 2, 9], device="cuda")
    logp, lse = prism.token_logprob(z, t)
    log = np.log
    assert np.allclose(_f64(logp), [-log(50), -inf, 0, -inf, -log(50), -2e4]) and np.allclose(_f64(lse), [log(50), -inf, 0, log(49), 1e4 + log(50), 1e4])
    d = prism.token_logprob_backward(torch.ones(6, device="cuda"), z, t, lse)
    ref = np.full((6, 50), -1 / 50)
    ref[1], ref[2], ref[3], ref[5] = 0, 0, -1 / 49, 0
    ref[2, 0], ref[3, 7], ref[5, 3] = -1, 0, -1
    for i, j in enumerate(t.tolist()):
        ref[i, j] += 1
    assert np.allclose(_f64(d), ref, atol=2e-3)                # lse of 1e4 is rounded by 5e-4
    r = prism.policy_loss(z[[0, 2, 4]], t[[0, 2, 4]])
    assert np.isclose(float(r.loss), 2 * log(50) / 3)
    # nothing to learn from
    r = prism.policy_loss(z, torch.full((6,), -1, device="cuda"))
    assert float(r.loss) == 0 and not any(bool(x.any()) for x in r[1:])
    r = prism.policy_loss(z[:0], t[:0])
    assert float(r.loss) == 0 and r.dlogits.shape == (0, 50)
    # a row of weight 0 may have any ratio
    w = torch.ones(6, device="cuda")
    w[5] = 0
    old = torch.zeros(6, device="cuda")
    old[5] = -1e30
    zz = z.clone()
    zz[1] = 0
    zz[3, 7] = 0
    r = prism.policy_loss(zz, t, advantages=-w, old_logp=old, weights=w)
    assert all(bool(x.isfinite().all()) for x in r) and not bool(r.dlogits[5].any())
    # where the ratio meets its bound the gradient is that of the ratio
    one = torch.zeros(1, 2, device="cuda")
    r = prism.policy_loss(one, t[:1], advantages=torch.ones(1, device="cuda"), old_logp=torch.full((1,), -log(2), device="cuda"), clip=(0.0, 0.0))
    assert abs(float(r.dlogp)) in (0.0, 1.0) and np.isclose(float(r.loss), -1.0)
    b = torch.randn(2, 3, 40, device="cuda")
    r = prism.policy_loss(b, torch.randint(0, 40, (2, 3), device="cuda"))
    assert r.logp.shape == (2, 3) and r.dlogits.shape == (2, 3, 40)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("v", [5, 300, 5000, 33000, 140000])
def test_logits_of_the_lowest_value(prism, dtype, v):
    """Masks of the type's lowest value: like any other logit, also where a row has no others; and rows far from zero."""
    low = torch.finfo(dtype).min
    g = torch.Generator().manual_seed(v)
    z = torch.randn(6, v, generator=g)
    z[0], z[1, 1:] = low, low
    z[2, ::2] = low
    z[3] = low
    z[3, 2:] = -float("inf")
    z[4] += 3e4
    z[5] = z[5].abs() * 1e37
    z = z.to(dtype).cuda()
    t = torch.tensor([v - 1, 0, 1, 1, 2, 3], device="cuda")
    logp, lse = prism.token_logprob(z, t)
    rlogp, rlse, p = R.logprob(_f64(z), t.tolist(), 1.0)
    # differences of logits are rounded to fp32, and a thread's sum of v / 64 terms
    off = E * np.where(p > 0, np.abs(np.where(p > 0, _f64(z), 0.0) - _f64(z).max(1, keepdims=True)) * p, 0.0).sum(1) * 3 + E * (v / 64 + 100)
    _close(logp, rlogp, off + 2 * E * np.abs(rlogp), "logp")
    _close(lse, rlse, off + E * np.abs(rlse), "lse")
    d = prism.token_logprob_backward(torch.ones(6, device="cuda"), z, t, lse)
    ref = R.logprob_gradient(np.ones(6), p, t.tolist(), 1.0)
    bound = _u(dtype) * np.abs(ref) + (off + 80 * E)[:, None] * p + 3 * E * (p + (ref > 0))
    _close(d, ref, bound, "dlogits")
    r = prism.policy_loss(z, t, weights=torch.ones(6, device="cuda"))
    _close(r.dlogits, -ref, bound, "dlogits in one pass")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [2.0 ** -100, 1e-6, 300.0, 2.0 ** 60])
def test_logits_scales_far_from_one(prism, dtype, scale):
    """Excluded logits stay excluded and probabilities are those of the scaled logits, whatever the scale."""
    g = torch.Generator().manual_seed(7)
    z = torch.randn(4, 700, generator=g)
    z[:, 3::5] = -float("inf")
    z[1] *= 1.0 / scale if scale < 1e10 else 1.0
    z[1, 3::5] = -float("inf")
    z = z.to(dtype).cuda()
    t = torch.tensor([0, 1, 2, 4], device="cuda")
    logp, lse = prism.token_logprob(z, t, scale=scale)
    rlogp, rlse, p = R.logprob(_f64(z), t.tolist(), scale)
    spread = scale * np.abs(np.where(p > 0, _f64(z), 0.0) - _f64(z).max(1, keepdims=True)) * p
    # three roundings of each exponent, a thread's sum and the joins; bf16 rounds the factor
    off = 4 * E * np.where(p > 0, spread, 0.0).sum(1) + 100 * E
    _close(logp, rlogp, off + 2 * E * np.abs(rlogp), "logp")
    _close(lse, rlse, off + 2 * E * np.abs(rlse), "lse")
    d = prism.policy_loss(z, t, scale=scale, weights=torch.ones(4, device="cuda")).dlogits
    ref = R.logprob_gradient(-np.ones(4), p, t.tolist(), scale)
    _close(d, ref, _u(dtype) * np.abs(ref) + scale * (4 * E * np.where(p > 0, spread, 0.0) + (off + 10 * E)[:, None] * p + 3 * E * (ref < 0)) + 1e-36, "dlogits")
    assert not bool(d[:, 3::5].any())


def test_offsets_past_32_bits(prism):
    """Rows that lie more than 2^31 elements behind the first."""
    n, width, stride = 40, 264, 1 << 26
    whole = torch.empty(n * stride, device="cuda", dtype=BF16).view(n, stride)          # 5 GB, the rows' beginnings only are touched
    out = torch.empty(n * stride, device="cuda", dtype=BF16).view(n, stride)[:, :width]
    x = whole[:, :width]
    x.copy_(torch.randn(n, width, generator=torch.Generator().manual_seed(1)))
    near, t = x.contiguous(), torch.arange(n - 1, -1, -1, device="cuda")
    assert torch.equal(prism.embedding(t, x, out=out), near[t])
    assert torch.equal(prism.embedding_backward(x, t, n, out=out), near[t])
    w = torch.ones(width, device="cuda")
    y, total, stats = prism.layer_norm(near, w, residual=near)
    got = prism.layer_norm(x, w, residual=x, out=(out, torch.empty_like(near)))
    assert torch.equal(got[0], y) and torch.equal(got[1], total) and torch.equal(got[2], stats)
    for a, b in zip(prism.layer_norm_backward(x, x, stats, w, dtotal=x, out=out), prism.layer_norm_backward(near, near, stats, w, dtotal=near)):
        assert torch.equal(a, b)
    logp, lse = prism.token_logprob(near, t)
    assert all(torch.equal(a, b) for a, b in zip(prism.token_logprob(x, t), (logp, lse)))
    assert torch.equal(prism.token_logprob_backward(logp, x, t, lse, out=out), prism.token_logprob_backward(logp, near, t, lse))
    assert all(torch.equal(a, b) for a, b in zip(prism.policy_loss(x, t, out=out), prism.policy_loss(near, t)))


def test_many_rows(prism):
    """More rows than one launch has workgroups for, and more tokens of one row than an unsigned count of 16 bits."""
    rows = (1 << 20) + 77
    z, t = torch.zeros(rows, 3, device="cuda"), torch.full((rows,), -1, device="cuda")
    z[-5:, 1], t[-5:] = 2.0, 1
    t[0] = 0
    logp, lse = prism.token_logprob(z, t)
    one = float(logp[-1])
    assert np.isclose(float(logp[0]), -np.log(3)) and np.isclose(one, 2 - np.log(2 + np.exp(2))) and bool((logp[1:-5] == 0).all()) and bool((logp[-5:] == one).all())
    r = prism.policy_loss(z, t)
    assert np.isclose(float(r.loss), -(float(logp[0]) + 5 * one) / 6) and not bool(r.dlogits[1:-5].any())
    assert torch.equal(r.logp, logp)
    y, _, _ = prism.layer_norm(z, eps=1.0)
    assert bool((y[:-5] == 0).all()) and bool((y[-5:] == y[-1]).all())
    d = prism.embedding_backward(torch.ones(rows, 2, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda"), 2)
    assert d.tolist() == [[rows, rows], [0, 0]]


def test_arrays_larger_than_the_caches(prism):
    """Their kernels read past the caches; rows (or columns) are the same bits as in calls of a part of them."""
    g = torch.Generator(device="cuda").manual_seed(1)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=BF16)   # noqa: E731
    for v in (32768, 65536, 131072, 66001):
        rows = (300 << 20) // (2 * v)
        z, t = make(rows, v), torch.randint(-1, v, (rows,), generator=g, device="cuda")
        w, old = torch.rand(rows, generator=g, device="cuda"), torch.full((rows,), -12.0, device="cuda")
        logp, lse = prism.token_logprob(z, t)
        r = prism.policy_loss(z, t, old_logp=old, weights=w)
        for a in (0, rows // 2, rows - 70):
            part = slice(a, a + 70)
            b = prism.policy_loss(z[part], t[part], old_logp=old[part], weights=w[part])
            assert torch.equal(r.dlogits[part], b.dlogits) and torch.equal(r.logp[part], b.logp)
            c = prism.token_logprob(z[part], t[part])
            assert torch.equal(logp[part], c[0]) and torch.equal(lse[part], c[1])
    for width in (768, 771, 4096, 4099, 8192):
        rows = (200 << 20) // (2 * width)
        x, res = make(rows, width), make(rows, width)
        weight = torch.rand(width, generator=g, device="cuda")
        y, total, stats = prism.layer_norm(x, weight, residual=res)
        dx, dw, db = prism.layer_norm_backward(y, total, stats, weight, dtotal=res)
        for a in (0, rows // 2, rows - 300):
            part = slice(a, a + 300)
            b = prism.layer_norm(x[part], weight, residual=res[part])
            assert all(torch.equal(p, q) for p, q in zip(b, (y[part], total[part], stats[part])))
            assert torch.equal(dx[part], prism.layer_norm_backward(y[part], total[part], stats[part], weight, dtotal=res[part])[0])
        n = (total.double() - stats[:, :1].double()) * stats[:, 1:].double()
        for got, terms in ((dw, y.double() * n), (db, y.double())):
            # a thread adds rows / 512 terms at most
            assert bool(((got.double() - terms.sum(0)).abs() <= (rows // 512 + 40) * E * terms.abs().sum(0)).all())
    n, rows, width = 70000, 20000, 1000
    dout, t = make(n, width), torch.randint(-1, rows, (n,), generator=g, device="cuda")
    d = prism.embedding_backward(dout, t, rows)
    assert torch.equal(d[:, :520], prism.embedding_backward(dout[:, :520], t, rows))          # (two pieces of 512 columns: tiles of the same length, the same sums)


def test_embedding_gradient_of_very_many_pieces(prism):
    """Tiles of more than 64 tokens: sums of ones are exact."""
    n, width = 600001, 65536
    t = (torch.rand(n, generator=torch.Generator().manual_seed(1)) < 0.3).int().cuda()
    d = prism.embedding_backward(torch.ones(1, width, device="cuda", dtype=BF16).expand(n, width), t, 2, scale=2.0 ** -10)
    ones = int(t.sum())
    want = (torch.tensor([n - ones, ones], device="cuda").float() * 2.0 ** -10).to(BF16)
    assert torch.equal(d, want.view(2, 1).expand(2, width))


# ------------------------------------------------------------------------------------------------------- streams and graphs

def _calls(prism, g, dtype):
    """Calls of every operator on arrays of their own, as functions without arguments."""
    tokens = torch.randint(-1, 300, (2000,), generator=g).cuda()
    table, x, r, w = _array(g, (300, 264), dtype), _array(g, (2000, 264), dtype), _array(g, (2000, 264), dtype), torch.rand(264, generator=g).cuda()
    z = _array(g, (60, 5003), dtype)
    t = torch.randint(-1, 5003, (60,), generator=g).cuda()
    old, adv = -torch.rand(60, generator=g).cuda(), torch.randn(60, generator=g).cuda()

    def ends():
        y, total, stats = prism.layer_norm(x, w, residual=r)
        logp, lse = prism.token_logprob(z, t)
        return (prism.embedding(tokens, table), prism.embedding_backward(x, tokens, 300), y, total, *prism.layer_norm_backward(x, total, stats, w, dtotal=r), logp, lse,
                prism.token_logprob_backward(adv, z, t, lse), *prism.policy_loss(z, t, advantages=adv, old_logp=old, ref_logp=old, kl=0.1), *prism.policy_loss(z, t, weights=adv))
    return ends, (x, r, z, table)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_ends_on_another_stream(prism, dtype):
    ends, _ = _calls(prism, torch.Generator().manual_seed(1), dtype)
    want = ends()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = ends()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_ends_in_graphs(prism, dtype):
    """Two graphs, replayed side by side on two streams, several times, on new inputs, with eager calls between."""
    made = [_calls(prism, torch.Generator().manual_seed(seed), dtype) for seed in (2, 3)]
    captured = []
    for ends, _ in made:
        ends()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = ends()
        captured.append((graph, out))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(4):
        for _, inputs in made:
            for x in inputs:
                x.mul_(0.75)
        want = [ends() for ends, _ in made]
        torch.cuda.synchronize()
        for s, (graph, _) in zip(streams, captured):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for w, (_, out) in zip(want, captured):
            assert all(torch.equal(a, b) for a, b in zip(w, out)), turn


def test_given_workspaces(prism):
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    d, t = torch.randn(500, 24, device="cuda"), torch.randint(0, 90, (500,), device="cuda")
    assert torch.equal(prism.embedding_backward(d, t, 90), prism.embedding_backward(d, t, 90, workspace=ws))
    with pytest.raises(prism.PrismError, match="workspace"):
        prism.embedding_backward(d, t, 90, workspace=ws[:100])
    y, total, stats = prism.layer_norm(d)
    assert all(torch.equal(a, b) for a, b in zip(prism.layer_norm_backward(d, total, stats), prism.layer_norm_backward(d, total, stats, workspace=ws)))
    with pytest.raises(prism.PrismError, match="workspace"):
        prism.layer_norm_backward(d, total, stats, workspace=ws[1:])
    z, t = torch.randn(9, 30, device="cuda"), torch.randint(0, 30, (9,), device="cuda")
    assert all(torch.equal(a, b) for a, b in zip(prism.policy_loss(z, t), prism.policy_loss(z, t, workspace=ws)))
    # without one the library keeps one for the stream
    desc = prism._pack(prism._EMBEDDING, 500, 90, 24, 1, 1.0, 24, 24, 0, 0)
    out = torch.empty(90, 24, device="cuda")
    u = torch.randint(0, 90, (500,), device="cuda")
    assert prism.lib().prism_embedding_backward(d.data_ptr(), u.data_ptr(), out.data_ptr(), prism.F32, desc, torch.cuda.current_stream().cuda_stream) == prism.OK
    assert torch.equal(out, prism.embedding_backward(d, u, 90))


def test_refusals_of_the_binding(prism):
    x, t = torch.randn(4, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    for call in (lambda: prism.embedding(t.float(), x), lambda: prism.embedding(t.cpu(), x), lambda: prism.embedding(t, x[0]), lambda: prism.embedding(t, x.half()),
                 lambda: prism.embedding(t, x.t()), lambda: prism.embedding(t, x, out=torch.empty(4, 7, device="cuda")), lambda: prism.embedding(t, x, scale=float("inf")),
                 lambda: prism.embedding(t, x, out=torch.empty(1, 8, device="cuda").expand(4, 8)), lambda: prism.embedding(t.expand(3, 4), x),
                 lambda: prism.embedding_backward(x, t[:3], 4), lambda: prism.embedding_backward(x, t, -1), lambda: prism.embedding_backward(x, t, 4, scale=1e50),
                 lambda: prism.layer_norm(x, weight=torch.ones(7, device="cuda")), lambda: prism.layer_norm(x, weight=x[0].bfloat16()), lambda: prism.layer_norm(x, eps=-1.0),
                 lambda: prism.layer_norm(x, residual=x[:3]), lambda: prism.layer_norm(x, out=(x, x)), lambda: prism.layer_norm(x, residual=x, out=(x, x)),
                 lambda: prism.layer_norm(torch.empty(2, 16385, device="cuda")), lambda: prism.layer_norm(x.permute(1, 0)), lambda: prism.layer_norm(x.cpu()),
                 lambda: prism.layer_norm_backward(x, x, torch.empty(3, 2, device="cuda")), lambda: prism.layer_norm_backward(x.bfloat16(), x, torch.empty(4, 2, device="cuda")),
                 lambda: prism.token_logprob(x, t[:3]), lambda: prism.token_logprob(x, t, scale=0.0), lambda: prism.token_logprob(x, t, scale=-1.0),
                 lambda: prism.token_logprob_backward(t, x, t, x[:, 0]), lambda: prism.policy_loss(x, t, kl=0.1), lambda: prism.policy_loss(x, t, kl=-0.1),
                 lambda: prism.policy_loss(x, t, clip=(1.5, 0.2)), lambda: prism.policy_loss(x, t, clip=(0.2, float("nan"))), lambda: prism.policy_loss(x, t, weights=t),
                 lambda: prism.policy_loss(x, t, gradient=False, out=x), lambda: prism.policy_loss(x, t, old_logp=x[:, 0])):
        with pytest.raises(prism.PrismError):
            call()
    assert not bool(torch.isnan(x).any())
