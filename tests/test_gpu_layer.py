"""The operators of a transformer layer (prism_dropout, prism_qk_norm_rope, prism_attention and their gradients) through the
C-ABI against the fp64 oracle.

Tolerances follow from what is rounded.  U is the relative error of one rounding to the type of the arrays (bf16 2^-8, fp32 2^-24).  Norm
and rotation round once; fp32 adds a few roundings of the arithmetic, counted at each test.  Attention rounds its results, and in bf16 the weights
and score gradients before their products: entry by entry the error is at most U (|result| + sum |weights| |values|) and what fp32 arithmetic adds to
the exponents."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import layer_ref as R

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


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
    assert np.all(np.isfinite(got)), what
    worst = np.max((np.abs(got - ref) - bound) if got.size else np.array([-1.0]))
    assert worst <= 0, (what, float(worst), float(np.max(np.abs(got - ref))))


# ---------------------------------------------------------------------------------------------------------------- dropout

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("n,shift", [(1, 0), (7, 0), (8, 0), (9, 1), (4099, 0), (70001, 3)])
def test_dropout(prism, dtype, residual, n, shift):
    g = torch.Generator().manual_seed(n)
    x = torch.randn(n + shift, generator=g).to(dtype).cuda()[shift:]
    r = (3.0 * torch.randn(n + shift, generator=g)).to(dtype).cuda()[shift:] if residual else None
    seed, offset, p = (5 << 40) + 77, 2 ** 32 - 3, 0.3
    y = prism.dropout(x, p, seed, offset=offset, residual=r)
    kept, factor = R.dropout_kept(0, n, p, seed, offset)
    ref = np.where(kept, _f64(x) * factor, 0.0) + (_f64(r) if residual else 0.0)
    # the result's rounding; fp32 arithmetic rounds the factor, the product and the sum
    extra = 3 * 2.0 ** -24 * (np.abs(_f64(x)) * factor + (np.abs(_f64(r)) if residual else 0.0))
    _close(y, ref, _u(dtype) * np.abs(ref) + extra, "dropout")
    assert torch.equal(y, prism.dropout(x, p, seed, offset=offset, residual=r))


def test_dropout_in_place_edges_and_nan(prism):
    x = torch.randn(1000, device="cuda").to(BF16)
    assert torch.equal(prism.dropout(x, 0.0, 1), x)
    y = x.clone()
    kept, factor = R.dropout_kept(0, 1000, 0.5, 9, 0)
    assert prism.dropout(y, 0.5, 9, out=y) is y and torch.equal(y, prism.dropout(x, 0.5, 9))
    z = torch.full((1000,), float("inf"), device="cuda")
    z[::2] = float("nan")
    out = _f64(prism.dropout(z, 0.5, 9))
    assert np.array_equal(np.isfinite(out), ~kept) and np.all(out[~kept] == 0)        # what is dropped is 0 whatever it held
    e = torch.empty(0, device="cuda")
    assert prism.dropout(e, 0.5, 9).numel() == 0


def test_dropout_past_32_bits_of_elements(prism):
    n = 2 ** 32 + 24
    x = torch.ones(n, dtype=BF16, device="cuda")
    prism.dropout(x, 0.5, 123, out=x)
    at = 2 ** 32 - 16
    kept, factor = R.dropout_kept(at, n - at, 0.5, 123, 0)
    assert np.array_equal(_f64(x[at:]), np.where(kept, factor, 0.0))
    first = R.dropout_kept(0, 40, 0.5, 123, 0)[0]
    assert not np.array_equal(first, kept)


def test_dropout_refusals(prism):
    x = torch.randn(64, device="cuda")
    for p in (-0.1, 1.0, 0.999995, float("nan")):
        with pytest.raises(prism.PrismError, match="PRISM_EINVAL"):
            prism.dropout(x, p, 1)
    for bad in (x[::2], x.to(torch.float16), x.cpu()):
        with pytest.raises(prism.PrismError):
            prism.dropout(bad, 0.1, 1)
    with pytest.raises(prism.PrismError):
        prism.dropout(x, 0.1, 1, residual=x[:32])
    L = prism.lib()
    assert L.prism_dropout(None, None, x.data_ptr(), 4, prism.F32, 0.1, 1, 0, None) == prism.EINVAL
    assert L.prism_dropout(x.data_ptr(), None, x.data_ptr(), -1, prism.F32, 0.1, 1, 0, None) == prism.EINVAL
    assert L.prism_dropout(x.data_ptr() + 2, None, x.data_ptr(), 4, prism.F32, 0.1, 1, 0, None) == prism.EINVAL
    assert L.prism_dropout(x.data_ptr(), None, x.data_ptr(), 4, 5, 0.1, 1, 0, None) == prism.EINVAL
    assert L.prism_dropout(None, None, None, 0, prism.F32, 0.1, 1, 0, None) == prism.OK


# ------------------------------------------------------------------------------------------------- norm and rotation

def _norm_rope_case(dtype, b, n, hq, hk, d, rot, seed, view):
    g = torch.Generator().manual_seed(seed)
    make = lambda h, s: (s * torch.randn(b, n, h, d, generator=g)).to(dtype).cuda()   # noqa: E731
    q, k, gq, gk = make(hq, 2.0), make(hk, 0.5), make(hq, 1.0), make(hk, 1.0)
    if view == "fused":
        both = torch.cat([q, k], 2).contiguous()
        q, k = both[:, :, :hq], both[:, :, hq:]
    elif view == "heads_first":
        q, k = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k))
    elif view == "odd":                                    # rows that no vector of 16 bytes fits
        q, k = (torch.cat([t, t[..., :1]], 3)[..., :d] for t in (q, k))
    pos = torch.randint(0, 200000, (b, n), generator=g, dtype=torch.int32)
    w = [(1.0 + 0.2 * torch.randn(d, generator=g)).cuda() for _ in range(2)]
    f = (10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64) / max(1, rot // 2))).float()
    return q, k, gq, gk, pos, w, f


NORM_ROPE = [
    # b, n, hq, hk, d, rot, interleaved, norm, view
    (1, 1, 1, 1, 64, 64, False, True, "plain"),
    (2, 5, 12, 12, 64, 64, False, True, "fused"),
    (2, 37, 8, 2, 128, 128, True, True, "heads_first"),
    (3, 7, 6, 3, 80, 40, True, True, "plain"),
    (1, 9, 4, 4, 80, 48, False, True, "plain"),
    (1, 9, 4, 4, 96, 32, False, False, "fused"),
    (2, 11, 3, 1, 33, 10, False, True, "plain"),
    (2, 11, 3, 1, 50, 50, True, True, "odd"),
    (1, 13, 2, 2, 64, 24, True, True, "odd"),
    (1, 6, 2, 1, 256, 256, False, True, "plain"),
    (1, 6, 2, 1, 256, 0, False, True, "plain"),
    (1, 3, 2, 1, 1, 0, False, True, "plain"),
    (4, 600, 16, 8, 64, 64, False, True, "plain"),
    (1, 3001, 32, 5, 128, 128, False, True, "plain"),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("b,n,hq,hk,d,rot,inter,norm,view", NORM_ROPE)
def test_norm_rope_and_gradients(prism, dtype, b, n, hq, hk, d, rot, inter, norm, view):
    q, k, gq, gk, pos, w, f = _norm_rope_case(dtype, b, n, hq, hk, d, rot, 7 * n + d, view)
    eps, scale = 1e-6, 1.25
    args = dict(inv_freq=f.cuda() if rot else None, positions=pos.cuda(), q_weight=w[0] if norm else None, k_weight=w[1] if norm else None, norm=norm,
                interleaved=inter, scale=scale, eps=eps)
    outs = prism.qk_norm_rope(q, k, **args)
    grads = prism.qk_norm_rope_backward(gq, gk, q, k, **args)
    again = prism.qk_norm_rope_backward(gq, gk, q, k, **args)
    assert all(torch.equal(x, y) for x, y in zip(grads, again) if x is not None)
    for x, g, wt, out, dx, dw in zip((q, k), (gq, gk), w, outs, grads[:2], grads[2:]):
        ref = lambda t, *a: R.norm_rope(t, pos.numpy(), f.double().numpy(), _f64(wt), norm, inter, scale, eps)   # noqa: E731
        x64, g64 = _f64(x), _f64(g)
        y = ref(x64)
        # fp32: mean of d squares, root and quotient, weight, sine and cosine (angle to 1e-7 rad at most, 2 units each), rotation: d / 8 + 24 roundings
        # of a row's largest entry at most
        arith = (d / 8 + 24) * 2.0 ** -24 * np.max(np.abs(y), axis=-1, keepdims=True) + 1e-30
        _close(out, y, _u(dtype) * np.abs(y) + arith, "out")
        rx, rw = R.norm_rope_grad(g64, x64, pos.numpy(), f.double().numpy(), _f64(wt), norm, inter, scale, eps)
        # dx: the same, on the two terms whose difference it is
        r = 1.0 / np.sqrt(np.mean(x64 * x64, -1, keepdims=True) + eps) if norm else 1.0
        dn = np.max(np.abs(g64), -1, keepdims=True) * 1.5 * scale * (np.max(np.abs(_f64(wt))) if norm else 1.0)
        size = r * dn * (1.0 + (np.max(np.abs(x64), -1, keepdims=True) ** 2 * r * r if norm else 0.0))
        _close(dx, rx, _u(dtype) * np.abs(rx) + (d / 8 + 24) * 2.0 ** -24 * size, "dx")
        if norm:
            # a sum of b n h terms in fp32, each off by a few units; partial sums of terms of random sign grow like the root of their number: 8 of it
            terms = 1.5 * scale * np.abs(g64).max() * np.max(np.abs(x64 * r))
            count = b * n * x.shape[2]
            _close(dw, rw, 2.0 ** -24 * terms * (8 * count ** 0.5 + 32 * count ** 0.5 + 32) * np.ones(d), "dw")
        else:
            assert dw is None


def test_norm_rope_one_of_two_in_place_and_start(prism):
    q, k, _, _, _, w, f = _norm_rope_case(BF16, 2, 19, 4, 2, 64, 64, 1, "plain")
    both = prism.qk_norm_rope(q, k, f.cuda(), start=1000, q_weight=w[0], k_weight=w[1])
    pos = (1000 + torch.arange(19, dtype=torch.int32)).repeat(2, 1).cuda()
    assert all(torch.equal(a, b) for a, b in zip(both, prism.qk_norm_rope(q, k, f.cuda(), positions=pos, q_weight=w[0], k_weight=w[1])))
    only, none = prism.qk_norm_rope(q, None, f.cuda(), start=1000, q_weight=w[0])
    assert none is None and torch.equal(only, both[0])
    none, only = prism.qk_norm_rope(None, k, f.cuda(), start=1000, k_weight=w[1])
    assert none is None and torch.equal(only, both[1])
    prism.qk_norm_rope(q, k, f.cuda(), start=1000, q_weight=w[0], k_weight=w[1], out=(q, k))
    assert torch.equal(q, both[0]) and torch.equal(k, both[1])
    e = torch.empty(0, 4, 2, 64, device="cuda", dtype=BF16)
    assert prism.qk_norm_rope(e, e, f.cuda())[0].shape == e.shape
    assert torch.all(prism.qk_norm_rope_backward(e, e, e, e, f.cuda())[2] == 0)


def test_norm_rope_zero_heads_and_row_of_zeros(prism):
    q = torch.zeros(1, 2, 1, 64, device="cuda")
    q[0, 1] = 1e-20
    y, _ = prism.qk_norm_rope(q, None, None, eps=1e-6)
    assert torch.all(torch.isfinite(y)) and torch.all(y[0, 0] == 0)


def test_norm_rope_refusals(prism):
    q = torch.randn(2, 3, 4, 64, device="cuda")
    f = torch.ones(32, device="cuda")
    bad = [dict(inv_freq=torch.ones(33, device="cuda")), dict(inv_freq=f.double()), dict(inv_freq=f, positions=torch.zeros(2, 4, dtype=torch.int32, device="cuda")),
           dict(inv_freq=f, eps=-1.0), dict(inv_freq=f, scale=float("inf")), dict(inv_freq=f, q_weight=torch.ones(63, device="cuda")),
           dict(inv_freq=f, norm=False, q_weight=torch.ones(64, device="cuda")), dict(inv_freq=f.cpu())]
    for kw in bad:
        with pytest.raises(prism.PrismError):
            prism.qk_norm_rope(q, q, **kw)
    with pytest.raises(prism.PrismError):
        prism.qk_norm_rope(None, None, f)
    with pytest.raises(prism.PrismError):
        prism.qk_norm_rope(q, q[:, :2], f)
    with pytest.raises(prism.PrismError, match="PRISM_EUNSUPPORTED"):
        prism.qk_norm_rope(torch.randn(1, 1, 1, 257, device="cuda"), None)
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    with pytest.raises(prism.PrismError, match="PRISM_ENOMEM"):
        prism.qk_norm_rope_backward(q, q, q, q, f, workspace=small)
    o = prism.NormRopeDesc()
    o.batch = o.len = o.q_heads = 1
    o.head_dim, o.rot_dim, o.scale = 8, 3, 1.0
    assert prism.lib().prism_qk_norm_rope(q.data_ptr(), None, q.data_ptr(), None, prism.F32, ctypes.byref(o), None) == prism.EINVAL
    o.rot_dim = 0
    assert prism.lib().prism_qk_norm_rope(q.data_ptr(), None, None, None, prism.F32, ctypes.byref(o), None) == prism.EINVAL
    assert prism.lib().prism_qk_norm_rope(q.data_ptr(), None, q.data_ptr(), None, prism.F32, None, None) == prism.EINVAL


# ---------------------------------------------------------------------------------------------------------- attention

def _heads(g, b, n, h, d, dtype, scale, view):
    t = (scale * torch.randn(b, n, h, d, generator=g)).to(dtype).cuda()
    if view == "heads_first":
        return t.transpose(1, 2).contiguous().transpose(1, 2)
    if view == "odd":
        return torch.cat([t, t[..., :1]], 3)[..., :d]
    if view == "wide":
        return torch.cat([t, t], 2)[:, :, :h]
    return t


def _check_attention(prism, dtype, b, n, m, hq, hk, d, view="plain", softcap=0.0, causal=False, slopes=None, prefix=None, k_lens=None, q_doc=None,
                     k_doc=None, train=True, seed=0, q_scale=1.5, scale=None, poison=False):
    g = torch.Generator().manual_seed(seed)
    q, k, v = _heads(g, b, n, hq, d, dtype, q_scale, view), _heads(g, b, m, hk, d, dtype, 1.0, view), _heads(g, b, m, hk, d, dtype, 1.0, view)
    dout = _heads(g, b, n, hq, d, dtype, 1.0, view)
    sc = d ** -0.5 if scale is None else scale
    arr = lambda x, t: None if x is None else torch.tensor(x, dtype=t).cuda()   # noqa: E731
    opt = dict(causal=causal, softcap=softcap, scale=sc, slopes=arr(slopes, F32), prefix=arr(prefix, torch.int32), k_lens=arr(k_lens, torch.int32),
               q_doc=arr(q_doc, torch.int32), k_doc=arr(k_doc, torch.int32))
    seen = [R.visible(n, m, causal, None if prefix is None else prefix[i], None if k_lens is None else k_lens[i], None if q_doc is None else q_doc[i],
                      None if k_doc is None else k_doc[i]) for i in range(b)]
    if poison:       # what nobody may look at: padding and what lies past a sequence's length
        for i in range(b):
            hidden_k = (np.asarray(k_doc[i]) < 0) if k_doc is not None else np.zeros(m, bool)
            if k_lens is not None:
                hidden_k = hidden_k | (np.arange(m) >= k_lens[i])
            for t, val in ((k, float("nan")), (v, float("inf"))):
                t[i, torch.from_numpy(hidden_k).cuda()] = val
            if q_doc is not None:
                for t in (q, dout):
                    t[i, torch.from_numpy(np.asarray(q_doc[i]) < 0).cuda()] = float("nan")
    out, lse = prism.attention(q, k, v, **opt)
    out2, lse2 = prism.attention(q, k, v, **opt)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    grads = prism.attention_backward(dout, q, k, v, out, lse, **opt) if train else ()
    if train:
        assert all(torch.equal(x, y) for x, y in zip(grads, prism.attention_backward(dout, q, k, v, out, lse, **opt)))
    u, G = _u(dtype), hq // hk
    Q, K, V, DO = (_f64(t) for t in (q, k, v, dout))
    ref = {x: np.zeros(s) for x, s in (("out", Q.shape), ("dq", Q.shape), ("dk", K.shape), ("dv", K.shape))}
    lim = {x: np.zeros(ref[x].shape) for x in ref}
    ref_lse, lim_lse = np.zeros((b, hq, n)), np.zeros((b, hq, n))
    for i in range(b):
        see, far = seen[i]
        for h in range(hq):
            kk, vv, qq, gg = (np.where(see.any(0)[:, None], K[i, :, h // G], 0), np.where(see.any(0)[:, None], V[i, :, h // G], 0),
                              np.where(see.any(1)[:, None], Q[i, :, h], 0), np.where(see.any(1)[:, None], DO[i, :, h], 0))
            r = R.attention_head(qq, kk, vv, see, far, sc, softcap, 0.0 if slopes is None else slopes[h], gg)
            # fp32 exponents: a dot product of d terms, the factors, the exponential; relative error of a weight.  (The 4: score, cap, bias and
            # reference are each rounded at their own size.)
            mag = sc * (np.abs(qq) @ np.abs(kk).T)
            worst = np.where(see, mag + (0.0 if slopes is None else slopes[h] * far), 0.0).max(initial=0.0) + softcap
            e32 = 2.0 ** -24 * ((d / 4 + 8) * worst + 4 * worst + np.sqrt(m) + 16)
            p, ds = r["p"], r["ds"]
            rel = (u if dtype == BF16 else 0.0) + 2 * e32
            lo = u * np.abs(r["out"]) + rel * (p @ np.abs(vv))
            ref["out"][i, :, h], lim["out"][i, :, h] = r["out"], lo + 1e-30
            ref_lse[i, h], lim_lse[i, h] = r["lse"], 2 * e32 + 2.0 ** -23 * np.where(np.isfinite(r["lse"]), np.abs(r["lse"]), 0.0)
            # score gradients: p (dp - D): dp a dot product in fp32, D from the rounded result
            adp = np.abs(gg) @ np.abs(vv).T
            dD = np.sum(np.abs(gg) * lo, 1, keepdims=True) + (d / 4 + 8) * 2.0 ** -24 * np.sum(np.abs(gg) * np.abs(r["out"]), 1, keepdims=True)
            eds = rel * np.abs(ds) + sc * p * (dD + (d / 4 + 8) * 2.0 ** -24 * adp) + 2 * e32 * sc * p * (adp + np.sum(np.abs(gg * r["out"]), 1, keepdims=True))
            ref["dq"][i, :, h], lim["dq"][i, :, h] = r["dq"], u * np.abs(r["dq"]) + eds @ np.abs(kk)
            ref["dk"][i, :, h // G] += r["dk"]
            lim["dk"][i, :, h // G] += eds.T @ np.abs(qq) + 1e-30
            ref["dv"][i, :, h // G] += r["dv"]
            lim["dv"][i, :, h // G] += rel * (p.T @ np.abs(gg)) + 1e-30
    lim["dk"] += u * np.abs(ref["dk"])
    lim["dv"] += u * np.abs(ref["dv"])
    _close(out, ref["out"], lim["out"], "out")
    got = _f64(lse)
    assert np.array_equal(np.isneginf(got), np.isneginf(ref_lse))
    fin = np.isfinite(ref_lse)
    assert np.all(np.abs(got[fin] - ref_lse[fin]) <= lim_lse[fin]), "lse"
    for x, t in zip(("dq", "dk", "dv"), grads):
        _close(t, ref[x], lim[x] + 1e-30, x)


def _slopes(h):
    return [2.0 ** (-8.0 * (i + 1) / h) for i in range(h)]


SIZES = [
    # n, m, hq, hk, d
    (1, 1, 1, 1, 64), (1, 70, 4, 1, 64), (5, 5, 2, 2, 32), (64, 64, 3, 3, 64), (65, 63, 2, 1, 64), (33, 129, 4, 2, 128),
    (129, 129, 2, 2, 128), (130, 257, 6, 2, 80), (257, 257, 2, 1, 96), (3, 300, 8, 2, 128), (70, 2, 2, 2, 64), (40, 0, 2, 1, 64),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n,m,hq,hk,d", SIZES)
def test_attention_sizes(prism, dtype, causal, n, m, hq, hk, d):
    _check_attention(prism, dtype, 2, n, m, hq, hk, d, causal=causal, seed=n + m)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("view,d", [("heads_first", 64), ("wide", 128), ("odd", 64), ("odd", 33), ("plain", 7), ("plain", 1), ("plain", 72), ("plain", 100)])
def test_attention_strides_and_head_sizes(prism, dtype, view, d):
    _check_attention(prism, dtype, 2, 67, 67, 4, 2, d, view=view, causal=True, softcap=5.0, slopes=_slopes(4), seed=d)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("softcap", [0.0, 3.0, 50.0])
@pytest.mark.parametrize("bias", [False, True])
def test_attention_cap_and_bias(prism, dtype, softcap, bias):
    _check_attention(prism, dtype, 1, 150, 150, 4, 2, 64, causal=True, softcap=softcap, slopes=_slopes(4) if bias else None, q_scale=6.0, seed=2)
    _check_attention(prism, dtype, 1, 70, 150, 4, 2, 64, softcap=softcap, slopes=_slopes(4) if bias else None, q_scale=6.0, seed=3)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [24, 32, 40, 65, 72, 80, 96, 104])
@pytest.mark.parametrize("softcap,bias", [(0.0, False), (0.0, True), (10.0, False), (10.0, True)])
def test_attention_widths_of_the_products(prism, dtype, d, softcap, bias):
    """Heads on both sides of every width that products come in; then few rows against many keys."""
    kw = dict(softcap=softcap, slopes=_slopes(4) if bias else None, q_scale=3.0)
    _check_attention(prism, dtype, 1, 203, 203, 4, 2, d, causal=True, seed=d, **kw)
    _check_attention(prism, dtype, 2, 3, 700, 4, 2, d, causal=True, k_lens=[700, 333], seed=d + 1, **kw)


def _docs(lengths, pad=0):
    return sum([[i] * x for i, x in enumerate(lengths)], []) + [-1] * pad


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_documents_and_rows_that_see_nothing(prism, dtype, causal):
    a, b = _docs([60, 4, 100, 1, 90], 20), _docs([1, 1, 200], 73)
    _check_attention(prism, dtype, 2, 275, 275, 4, 2, 64, causal=causal, q_doc=[a, b], k_doc=[a, b], seed=5, poison=True)
    rng = np.random.default_rng(1)       # in no order, some queries of documents without keys
    q, k = rng.integers(-1, 6, (2, 140)).tolist(), rng.integers(-1, 4, (2, 200)).tolist()
    _check_attention(prism, dtype, 2, 140, 200, 2, 2, 32, causal=causal, q_doc=q, k_doc=k, seed=6, poison=True)
    none = [[-1] * 30, [3] * 30]
    _check_attention(prism, dtype, 2, 30, 30, 2, 1, 64, causal=causal, q_doc=none, k_doc=[[2] * 30, [4] * 30], seed=7, poison=True)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_prefix_and_lengths(prism, dtype):
    _check_attention(prism, dtype, 4, 150, 150, 2, 2, 64, causal=True, prefix=[0, 1, 70, 150], seed=8, slopes=_slopes(2))
    _check_attention(prism, dtype, 4, 40, 150, 2, 1, 64, causal=True, prefix=[200, 0, 64, 3], k_lens=[150, 40, 20, 0], seed=9, poison=True)
    _check_attention(prism, dtype, 4, 3, 300, 8, 2, 128, k_lens=[300, 1, 65, -5], seed=10, poison=True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("docs", [False, True])
def test_attention_in_parts(prism, dtype, causal, docs):
    """Few rows against many keys (forward, dq) and few keys against many rows (dk, dv): split and joined."""
    kw = dict(q_doc=[[1] * 7], k_doc=[_docs([500, 900], 100)]) if docs else {}
    _check_attention(prism, dtype, 1, 7, 1500, 4, 1, 64, causal=causal, seed=11, poison=True, **kw)
    kw = dict(k_doc=[[1] * 7], q_doc=[_docs([500, 900], 100)]) if docs else {}
    _check_attention(prism, dtype, 1, 1500, 7, 4, 1, 64, seed=12, poison=True, **kw)
    _check_attention(prism, dtype, 3, 1, 2000, 4, 2, 128, causal=causal, k_lens=[2000, 0, 130], softcap=20.0, train=False, seed=13, poison=True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n,m", [(1, 1), (5, 300), (70, 400), (300, 20)])
def test_attention_keys_whose_documents_no_query_has(prism, dtype, causal, n, m):
    """Key tiles without rows, the first sequence's too: nothing lies before its documents."""
    q_doc, k_doc = [[1] * n, [2] * n], [[7] * m, [2] * (m // 2) + [9] * (m - m // 2)]
    _check_attention(prism, dtype, 2, n, m, 4, 2, 64, causal=causal, q_doc=q_doc, k_doc=k_doc, seed=17)


def test_attention_large_scores_stay_finite(prism):
    _check_attention(prism, F32, 1, 40, 200, 1, 1, 64, q_scale=200.0, seed=14, train=False)
    _check_attention(prism, BF16, 1, 40, 200, 1, 1, 64, q_scale=200.0, seed=15, train=False)


def test_attention_rows_grow_late(prism):
    """Scores that grow along the keys: the running maximum moves at every tile."""
    n, m, d = 32, 640, 64
    q = torch.ones(1, n, 1, d, device="cuda")
    k = (torch.arange(m, device="cuda").float() / 8)[None, :, None, None].expand(1, m, 1, d).contiguous()
    v = torch.randn(1, m, 1, d, device="cuda")
    out, lse = prism.attention(q, k, v, scale=1.0 / d)
    s = torch.arange(m, dtype=torch.float64) / 8
    ref = torch.softmax(s, 0) @ v[0, :, 0].double().cpu()
    assert torch.allclose(out[0, :, 0].double().cpu(), ref.expand(n, d), atol=2e-4, rtol=0)      # exponents up to 80 in fp32: 80 * 2^-22 of values up to 5
    assert torch.allclose(lse.double().cpu(), torch.logsumexp(s, 0).expand(1, 1, n), atol=2e-5, rtol=0)


def test_attention_offsets_past_32_bits(prism):
    """Keys whose offsets pass 2^32 bytes and 2^32 elements."""
    m, gap, d = 4200, 1 << 20, 64
    big = torch.empty(m * gap + d, dtype=BF16, device="cuda")
    k = torch.as_strided(big, (1, m, 1, d), (m * gap, gap, d, 1))
    v = torch.as_strided(big, (1, m, 1, d), (m * gap, gap, d, 1), storage_offset=d * 2)
    g = torch.Generator().manual_seed(3)
    kc, vc, q = (torch.randn(1, x, 1, d, generator=g).to(BF16).cuda() for x in (m, m, 2))
    k.copy_(kc)
    v.copy_(vc)
    for kw in (dict(), dict(causal=True)):
        a, b = prism.attention(q, k, v, **kw), prism.attention(q, kc, vc, **kw)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    do = torch.randn(1, 2, 1, d, generator=g).to(BF16).cuda()
    x, y = prism.attention_backward(do, q, k, v, *a, causal=True), prism.attention_backward(do, q, kc, vc, *a, causal=True)
    assert all(torch.equal(s, t) for s, t in zip(x, y))


def test_attention_other_stream_and_given_workspace(prism):
    g = torch.Generator().manual_seed(4)
    q, k, v = (torch.randn(1, 9, 2, 64, generator=g).cuda(), torch.randn(1, 3000, 2, 64, generator=g).cuda(), torch.randn(1, 3000, 2, 64, generator=g).cuda())
    ref, lse = prism.attention(q, k, v)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        out, _ = prism.attention(q, k, v)
    s.synchronize()
    assert torch.equal(out, ref)
    o = prism.AttentionDesc.from_buffer_copy(prism._attention_desc(q, k, v, q, (), None, False, 0.0, None, None, None, None, None, None)[1])
    need = ctypes.c_size_t(0)
    assert prism.lib().prism_attention_workspace_bytes(prism.F32, ctypes.byref(o), 0, ctypes.byref(need)) == prism.OK and need.value > 0
    ws = torch.empty(need.value, dtype=torch.uint8, device="cuda")
    assert torch.equal(prism.attention(q, k, v, workspace=ws)[0], ref)
    with pytest.raises(prism.PrismError, match="PRISM_ENOMEM"):
        prism.attention(q, k, v, workspace=ws[:256])


def test_layer_calls_in_a_graph(prism):
    """Captured after one eager call, replayed several times on new contents with eager work between."""
    g = torch.Generator(device="cuda").manual_seed(5)
    new = lambda: [torch.randn(1, 200, 2, 64, device="cuda", generator=g) for _ in range(4)]   # noqa: E731
    q, k, v, do = new()
    doc = torch.tensor([_docs([50, 100], 50)], dtype=torch.int32).cuda()
    f = torch.ones(32, device="cuda")

    def step(q, k, v, do):
        a, b = prism.qk_norm_rope(q, k, f)
        out, lse = prism.attention(a, b, v, causal=True, q_doc=doc, k_doc=doc)
        da, db, dv = prism.attention_backward(do, a, b, v, out, lse, causal=True, q_doc=doc, k_doc=doc)
        return (prism.dropout(out, 0.2, 7, residual=q), dv) + prism.qk_norm_rope_backward(da, db, q, k, f)
    step(q, k, v, do)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(q, k, v, do)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        outs = step(q, k, v, do)
    for _ in range(4):
        for t, x in zip((q, k, v, do), new()):
            t.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        assert all(torch.equal(a, b) for a, b in zip(got, step(q, k, v, do)))
        torch.cuda.synchronize()


def test_attention_backward_without_queries(prism):
    q, k = torch.empty(1, 0, 2, 64, device="cuda"), torch.randn(1, 9, 2, 64, device="cuda")
    out, lse = prism.attention(q, k, k)
    dq, dk, dv = prism.attention_backward(q, q, k, k, out, lse)
    assert dq.numel() == 0 and torch.all(dk == 0) and torch.all(dv == 0)


def test_attention_refusals(prism):
    q, k = torch.randn(2, 3, 4, 64, device="cuda"), torch.randn(2, 5, 2, 64, device="cuda")
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")   # noqa: E731
    bad = [dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(softcap=-1.0), dict(softcap=float("inf")), dict(prefix=i32(2)), dict(q_doc=i32(2, 3)),
           dict(q_doc=i32(2, 3), k_doc=i32(2, 4)), dict(k_lens=i32(3)), dict(slopes=torch.ones(2, device="cuda")), dict(k_lens=i32(2).long()),
           dict(slopes=torch.ones(4))]
    for kw in bad:
        with pytest.raises(prism.PrismError):
            prism.attention(q, k, k, **kw)
    for a, b, c in ((q[:, :, :3], k, k), (q, k, k[:, :4]), (q, k.to(BF16), k), (q[..., ::2], k[..., ::2], k[..., ::2]), (q[0], k[0], k[0]), (q.cpu(), k, k)):
        with pytest.raises(prism.PrismError):
            prism.attention(a, b, c)
    with pytest.raises(prism.PrismError, match="PRISM_EUNSUPPORTED"):
        prism.attention(*(torch.randn(1, 2, 1, 129, device="cuda") for _ in range(3)))
    out, lse = prism.attention(q, k, k)
    with pytest.raises(prism.PrismError):
        prism.attention_backward(out, q, k, k, out, lse[:, :, :2])
    L = prism.lib()
    o = prism.AttentionDesc.from_buffer_copy(prism._attention_desc(q, k, k, q, (), None, False, 0.0, None, None, None, None, None, None)[1])
    assert L.prism_attention(q.data_ptr(), k.data_ptr(), None, q.data_ptr(), None, prism.F32, ctypes.byref(o), None) == prism.EINVAL
    assert L.prism_attention(q.data_ptr(), k.data_ptr(), k.data_ptr(), q.data_ptr(), None, 9, ctypes.byref(o), None) == prism.EINVAL
    o.q_heads = 3
    assert L.prism_attention(q.data_ptr(), k.data_ptr(), k.data_ptr(), q.data_ptr(), None, prism.F32, ctypes.byref(o), None) == prism.EINVAL
    assert "multiple" in L.prism_last_error().decode()
    o.q_heads, o.q.token = 4, -1
    assert L.prism_attention(q.data_ptr(), k.data_ptr(), k.data_ptr(), q.data_ptr(), None, prism.F32, ctypes.byref(o), None) == prism.EINVAL
    o.q.token = 256
    o.q_heads, o.batch, o.k_len = 4, 1 << 20, 1 << 20
    assert L.prism_attention(q.data_ptr(), k.data_ptr(), k.data_ptr(), q.data_ptr(), None, prism.F32, ctypes.byref(o), None) == prism.EUNSUPPORTED


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("view", ["plain", "heads_first"])
@pytest.mark.parametrize("group", [3, 5, 8, 16, 32, 64])
@pytest.mark.parametrize("d", [64, 80, 128])
def test_attention_groups_of_heads(prism, dtype, view, group, d):
    """Groups on both sides of the rows of a tile and of the rows between a thread's chunks, two of them, several whole tiles and a part of one."""
    _check_attention(prism, dtype, 2, 37, 45, 2 * group, 2, d, view=view, causal=True, seed=group)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("n,m,d", [(90, 90, 64), (70, 150, 80), (70, 150, 128), (3, 700, 128)])
@pytest.mark.parametrize("softcap", [500.0, 3e4, 1e6, 1e9])
def test_attention_caps_far_above_the_scores(prism, dtype, bias, n, m, d, softcap):
    """A cap far above the scores leaves them almost as they are: their error is some units of themselves, whatever the cap."""
    g = torch.Generator().manual_seed(21)
    q, k, v, do = (_heads(g, 1, x, h, d, dtype, s, "plain") for x, h, s in ((n, 2, 3.0), (m, 1, 1.0), (m, 1, 1.0), (n, 2, 1.0)))
    sl = _slopes(2) if bias else [0.0, 0.0]
    opt = dict(causal=True, softcap=softcap, scale=d ** -0.5, slopes=torch.tensor(sl, device="cuda") if bias else None)
    out, lse = prism.attention(q, k, v, **opt)
    grads = prism.attention_backward(do, q, k, v, out, lse, **opt)
    see, far = R.visible(n, m, True)
    K, V, u = _f64(k)[0, :, 0], _f64(v)[0, :, 0], _u(dtype)
    total = {x: 0.0 for x in ("dk", "dv", "lim_dk", "lim_dv")}
    for h in range(2):
        Q, G = _f64(q)[0, :, h], _f64(do)[0, :, h]
        r = R.attention_head(Q, K, V, see, far, d ** -0.5, softcap, sl[h], G)
        mag = d ** -0.5 * (np.abs(Q) @ np.abs(K).T)
        # a score: a product of d terms, scaling, tanh, cap, bias and reference, some units of its size each, and the plain tanh's 2^-23 of a cap of 1024 at most
        e = 2.0 ** -24 * ((d / 4 + 24) * (mag + sl[h] * far).max(where=see, initial=0.0) + np.sqrt(m) + 16) + (2.0 ** -23 * min(softcap, 1024.0))
        p, rel = r["p"], (u if dtype == BF16 else 0.0) + 2 * e
        lo = u * np.abs(r["out"]) + rel * (p @ np.abs(V))
        adp, ago = np.abs(G) @ np.abs(V).T, np.sum(np.abs(G * r["out"]), 1, keepdims=True)
        dD = np.sum(np.abs(G) * lo, 1, keepdims=True) + (d / 4 + 8) * 2.0 ** -24 * ago
        eds = rel * np.abs(r["ds"]) + d ** -0.5 * p * (dD + (d / 4 + 8) * 2.0 ** -24 * adp + 2 * e * (adp + ago))
        _close(out[0, :, h], r["out"], lo, "out")
        assert np.max(np.abs(_f64(lse)[0, h] - r["lse"])) <= 2 * e + 2.0 ** -23 * np.abs(r["lse"]).max()
        _close(grads[0][0, :, h], r["dq"], u * np.abs(r["dq"]) + eds @ np.abs(K), "dq")
        for x, t, lim in (("dk", r["dk"], eds.T @ np.abs(Q)), ("dv", r["dv"], rel * (p.T @ np.abs(G)))):
            total[x] = total[x] + t
            total["lim_" + x] = total["lim_" + x] + lim
    _close(grads[1][0, :, 0], total["dk"], u * np.abs(total["dk"]) + total["lim_dk"] + 1e-30, "dk")
    _close(grads[2][0, :, 0], total["dv"], u * np.abs(total["dv"]) + total["lim_dv"] + 1e-30, "dv")


def _queries_that_see_nothing(why, n, m):
    """(mask arguments of three sequences, which queries see no key)."""
    if why == "lengths":          # queries before the first key
        lens = [m, n // 3, 0]
        return dict(causal=True, k_lens=torch.tensor(lens, dtype=torch.int32).cuda()), [R.visible(n, m, True, keys=x)[0].any(1) for x in lens]
    q = [[0] * (n // 2) + [5] * (n - n // 2), [7] * n, (_docs([n // 4] * 4) + [1] * n)[:n]]      # documents that have no key
    k = [[0] * m, [2] * m, ([0] * (m // 2) + [3] * m)[:m]]
    arr = lambda x: torch.tensor(x, dtype=torch.int32).cuda()   # noqa: E731
    return dict(q_doc=arr(q), k_doc=arr(k)), [R.visible(n, m, q_doc=q[i], k_doc=k[i])[0].any(1) for i in range(3)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("why", ["lengths", "documents"])
@pytest.mark.parametrize("softcap,bias", [(0.0, False), (20.0, True)])
@pytest.mark.parametrize("n,m,hq,d", [(200, 200, 4, 64), (300, 300, 2, 128), (130, 1100, 6, 64), (9, 90, 2, 80), (40, 40, 32, 128)])
def test_attention_queries_that_see_nothing_may_hold_anything(prism, dtype, why, softcap, bias, n, m, hq, d):
    """The same bits, gradients too, whatever is in queries without a key and in their dout."""
    g = torch.Generator().manual_seed(23)
    mask, some = _queries_that_see_nothing(why, n, m)
    q, k, v, do = (_heads(g, 3, x, h, d, dtype, 1.0, "plain") for x, h in ((n, hq), (m, 2), (m, 2), (n, hq)))
    opt = dict(softcap=softcap, slopes=torch.tensor(_slopes(hq), device="cuda") if bias else None, **mask)
    none = torch.from_numpy(~np.stack(some)).cuda()
    assert bool(none.any()) and not bool(none.all())
    results = []
    for x in (0.0, float("nan"), float("inf")):
        a, b = q.clone(), do.clone()
        a[none], b[none] = x, x
        out, lse = prism.attention(a, k, v, **opt)
        results.append((out, lse) + prism.attention_backward(b, a, k, v, out, lse, **opt))
    assert torch.all(results[0][0][none] == 0) and torch.all(results[0][2][none] == 0)
    assert torch.all(torch.isneginf(results[0][1].transpose(1, 2)) == none[:, :, None])
    for r in results[1:]:
        for x, y, what in zip(results[0], r, ("out", "lse", "dq", "dk", "dv")):
            assert torch.equal(x, y), what


@pytest.mark.parametrize("norm", [True, False])
def test_norm_rope_gradients_of_one_of_two(prism, norm):
    q, k, gq, gk, pos, w, f = _norm_rope_case(F32, 2, 19, 4, 2, 64, 32, 1, "plain")
    args = dict(inv_freq=f.cuda(), positions=pos.cuda(), norm=norm)
    w = w if norm else (None, None)
    both = prism.qk_norm_rope_backward(gq, gk, q, k, q_weight=w[0], k_weight=w[1], **args)
    dq, dk, dqw, dkw = prism.qk_norm_rope_backward(gq, None, q, None, q_weight=w[0], **args)
    assert torch.equal(dq, both[0]) and dk is None and dkw is None and (torch.equal(dqw, both[2]) if norm else dqw is None)
    dq, dk, dqw, dkw = prism.qk_norm_rope_backward(None, gk, None, k, k_weight=w[1], **args)
    assert torch.equal(dk, both[1]) and dq is None and dqw is None and (torch.equal(dkw, both[3]) if norm else dkw is None)
    e = torch.empty(0, 4, 2, 64, device="cuda")
    assert (prism.qk_norm_rope_backward(e, None, e, None, norm=norm)[2] is None) == (not norm)


def test_numbers_that_no_description_holds(prism):
    q, k, f = torch.randn(1, 3, 2, 64, device="cuda"), torch.randn(1, 5, 2, 64, device="cuda"), torch.ones(32, device="cuda")
    for kw in (dict(start=2 ** 31), dict(start=2 ** 31 - 2), dict(scale=1e39), dict(eps=1e39)):
        with pytest.raises(prism.PrismError):
            prism.qk_norm_rope(q, None, f, **kw)
    prism.qk_norm_rope(q, None, f, start=2 ** 31 - 3)
    for kw in (dict(scale=1e39), dict(softcap=1e39)):
        with pytest.raises(prism.PrismError):
            prism.attention(q, k, k, **kw)
