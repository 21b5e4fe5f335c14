"""The layer operators' checks and workspace sizes, and the frequencies of the rotation: what needs no GPU.  Pointers handed over here are never read: every call is
refused, or empty, before anything is enqueued."""
import ctypes
import os

import numpy as np
import pytest

ADDRESS = 1 << 20


@pytest.fixture(scope="module")
def prism():
    from paper_2601_22137_amd import build, prism as P
    if not os.path.exists(P.LIB_PATH):
        build.build(verbose=False)
    P.lib()
    return P


def _attention(prism, **kw):
    d = prism.AttentionDesc()
    size = dict(batch=2, q_len=64, k_len=64, q_heads=4, k_heads=2, head_dim=64, scale=0.125)
    size.update(kw)
    for k, v in size.items():
        setattr(d, k, v)
    return d


def _bytes(prism, d, backward, dtype=None):
    out = ctypes.c_size_t(1)
    rc = prism.lib().prism_attention_workspace_bytes(prism.BF16 if dtype is None else dtype, ctypes.byref(d), backward, ctypes.byref(out))
    return rc, out.value


@pytest.mark.parametrize("kw", [dict(batch=-1), dict(q_len=-1), dict(k_len=-1), dict(head_dim=0), dict(q_heads=3), dict(k_heads=0), dict(q_heads=0), dict(scale=0.0),
                                dict(scale=-1.0), dict(scale=float("inf")), dict(softcap=-1.0), dict(softcap=float("nan")), dict(q_doc=ADDRESS), dict(k_doc=ADDRESS),
                                dict(prefix=ADDRESS)])
def test_attention_refuses(prism, kw):
    d = _attention(prism, **kw)
    assert prism.lib().prism_attention(ADDRESS, ADDRESS, ADDRESS, ADDRESS, None, prism.BF16, ctypes.byref(d), None) == prism.EINVAL
    assert prism.lib().prism_attention_backward(*[ADDRESS] * 9, prism.BF16, ctypes.byref(d), None) == prism.EINVAL
    assert _bytes(prism, d, 0)[0] == prism.EINVAL
    assert prism.lib().prism_last_error()


def test_attention_refuses_pointers_and_sizes(prism):
    L, d = prism.lib(), _attention(prism)
    for args in ((None, ADDRESS, ADDRESS, ADDRESS), (ADDRESS, None, ADDRESS, ADDRESS), (ADDRESS, ADDRESS, None, ADDRESS), (ADDRESS, ADDRESS, ADDRESS, None),
                 (ADDRESS + 1, ADDRESS, ADDRESS, ADDRESS)):
        assert L.prism_attention(*args, None, prism.BF16, ctypes.byref(d), None) == prism.EINVAL
    assert L.prism_attention(*[ADDRESS] * 4, None, 9, ctypes.byref(d), None) == prism.EINVAL
    assert L.prism_attention(*[ADDRESS] * 4, None, prism.BF16, None, None) == prism.EINVAL
    for kw in (dict(head_dim=129), dict(q_len=1 << 30, q_heads=8), dict(k_len=1 << 30), dict(batch=1 << 24, k_len=1 << 10)):
        assert _bytes(prism, _attention(prism, **kw), 0)[0] == prism.EUNSUPPORTED
    d.v.head = -64
    assert L.prism_attention(*[ADDRESS] * 4, None, prism.BF16, ctypes.byref(d), None) == prism.EINVAL


def test_empty_calls_touch_nothing(prism):
    L = prism.lib()
    for kw in (dict(batch=0), dict(q_len=0), dict(q_heads=0, k_heads=0)):
        assert L.prism_attention(None, None, None, None, None, prism.BF16, ctypes.byref(_attention(prism, **kw)), None) == prism.OK
    assert L.prism_attention_backward(*[None] * 9, prism.BF16, ctypes.byref(_attention(prism, q_len=0, k_len=0)), None) == prism.OK
    o = prism.NormRopeDesc()
    o.batch, o.len, o.head_dim, o.scale = 2, 0, 64, 1.0
    assert L.prism_qk_norm_rope(None, None, None, None, prism.BF16, ctypes.byref(o), None) == prism.OK
    assert L.prism_dropout(None, None, None, 0, prism.F32, 0.5, 0, 0, None) == prism.OK


def test_workspaces(prism):
    """None where a call is one launch; the parts of a few rows' keys; the gradients' row sums and parts, within a bound that does not grow with the square of
    the length."""
    full = _attention(prism, batch=8, q_len=8192, k_len=8192, q_heads=32, k_heads=8, head_dim=128, causal=1)
    assert _bytes(prism, full, 0) == (prism.OK, 0)
    one = _attention(prism, batch=1, q_len=1, k_len=32768, q_heads=8, k_heads=8, head_dim=128)
    rc, size = _bytes(prism, one, 0)
    assert rc == prism.OK and 8 * 128 * 4 < size <= 64 * 8 * (128 + 2) * 4 + 512
    for dtype in (prism.F32, prism.BF16):
        for n in (1, 63, 1000, 4096, 8192):
            d = _attention(prism, q_len=n, k_len=n, causal=1)
            rc, size = _bytes(prism, d, 1, dtype)
            # row sums; at most as many parts as fill 1024 workgroups of 128 keys, two fp32 arrays of a head each, and 64 of a short row tile's dq
            assert rc == prism.OK and 2 * 4 * n * 2 * 4 <= size <= 16 * n * 8 + 2 * 64 * 64 * 4 * 4 * max(n, 128) * 4 + 2048
    docs = _attention(prism, q_doc=ADDRESS, k_doc=ADDRESS)
    assert _bytes(prism, docs, 1)[1] > _bytes(prism, _attention(prism), 1)[1]
    o, out = prism.NormRopeDesc(), ctypes.c_size_t(0)
    o.batch, o.len, o.q_heads, o.k_heads, o.head_dim, o.rot_dim, o.scale, o.norm = 1, 100, 4, 2, 64, 0, 1.0, 1
    assert prism.lib().prism_norm_rope_workspace_bytes(prism.BF16, ctypes.byref(o), ctypes.byref(out)) == prism.OK and out.value > 0
    o.head_dim = 257
    assert prism.lib().prism_norm_rope_workspace_bytes(prism.BF16, ctypes.byref(o), ctypes.byref(out)) == prism.EUNSUPPORTED


@pytest.mark.parametrize("kw", [dict(rot_dim=3), dict(rot_dim=66), dict(rot_dim=-2), dict(rot_dim=4), dict(scale=float("nan")), dict(norm=1, eps=-1.0), dict(head_dim=0),
                                dict(q_weight=ADDRESS), dict(len=-1)])
def test_norm_rope_refuses(prism, kw):
    o = prism.NormRopeDesc()
    size = dict(batch=1, len=4, q_heads=2, k_heads=1, head_dim=64, scale=1.0)
    size.update(kw)
    for k, v in size.items():
        setattr(o, k, v)
    assert prism.lib().prism_qk_norm_rope(*[ADDRESS] * 4, prism.F32, ctypes.byref(o), None) == prism.EINVAL
    assert prism.lib().prism_qk_norm_rope_backward(*[ADDRESS] * 8, prism.F32, ctypes.byref(o), None) == prism.EINVAL


@pytest.mark.parametrize("p", [-0.1, 1.0, 2.0, 0.999995, float("nan")])
def test_dropout_refuses(prism, p):
    assert prism.lib().prism_dropout(ADDRESS, None, ADDRESS, 8, prism.F32, p, 1, 0, None) == prism.EINVAL


def test_frequencies(prism):
    f, s = prism.rope_frequencies(64)
    assert s == 1.0 and np.allclose(f.numpy(), 10000.0 ** (-np.arange(32) / 32), rtol=1e-6)
    g, _ = prism.rope_frequencies(64, scaling="linear", factor=4.0)
    assert np.allclose(g.numpy() * 4, f.numpy(), rtol=1e-6)
    g, _ = prism.rope_frequencies(64, scaling="base", factor=4.0)
    assert np.isclose(g[0], f[0]) and np.isclose(g[-1] * 4, f[-1], rtol=1e-5) and np.all(np.diff(g.numpy()) < 0)
    g, s = prism.rope_frequencies(64, scaling="by_turns", factor=8.0, original_len=4096)
    turns = 4096 * f.numpy() / (2 * np.pi)
    assert np.allclose(g.numpy()[turns > 32], f.numpy()[turns > 32]) and np.allclose(g.numpy()[turns < 1] * 8, f.numpy()[turns < 1], rtol=1e-6)
    assert np.isclose(s, 0.1 * np.log(8.0) + 1.0)
    for bad in (dict(rot_dim=3), dict(rot_dim=0), dict(rot_dim=8, factor=0.0), dict(rot_dim=8, scaling="none"), dict(rot_dim=8, scaling="by_turns", factor=2.0)):
        with pytest.raises(prism.PrismError):
            prism.rope_frequencies(**bad)


@pytest.mark.parametrize("kw", [dict(scale=3e38), dict(softcap=3e38), dict(softcap=1e-39), dict(softcap=1e-38, scale=10.0), dict(softcap=1e30, scale=1e-9)])
def test_attention_refuses_factors_that_leave_fp32(prism, kw):
    """Scores are taken times scale log2(e), or scale / softcap and softcap log2(e): an infinity there gives NaN for scores of 0, a subnormal loses digits."""
    d = _attention(prism, **kw)
    assert _bytes(prism, d, 0)[0] == prism.EINVAL and _bytes(prism, d, 1)[0] == prism.EINVAL
    assert b"softcap" in prism.lib().prism_last_error()
    for kw in (dict(scale=1e37), dict(scale=1e-40), dict(softcap=1e37), dict(softcap=1e-30)):
        assert _bytes(prism, _attention(prism, **kw), 0)[0] == prism.OK


def test_grids_that_no_launch_takes_are_refused_by_the_check(prism):
    """A launch takes fewer than 2^32 work-items."""
    most = dict(batch=(1 << 23) - 1, q_len=1, k_len=16, q_heads=2, k_heads=2)
    for back in (0, 1):
        assert _bytes(prism, _attention(prism, **most), back)[0] == prism.OK
        assert _bytes(prism, _attention(prism, **dict(most, batch=1 << 23)), back)[0] == prism.EUNSUPPORTED
    o = prism.NormRopeDesc()
    o.batch, o.len, o.q_heads, o.head_dim, o.scale = 1 << 20, 1, 1030, 40, 1.0
    o.q.batch, o.q.token, o.q.head = 1030 * 41, 1030 * 41, 41               # (rows of no whole vectors: a work-item for 16 entries)
    o.q_out = o.q
    assert prism.lib().prism_qk_norm_rope(ADDRESS, None, ADDRESS, None, prism.BF16, ctypes.byref(o), None) == prism.EUNSUPPORTED


def test_positions_past_32_bits_are_refused(prism):
    o = prism.NormRopeDesc()
    o.batch, o.len, o.q_heads, o.head_dim, o.scale, o.start = 1, 3, 1, 8, 1.0, 2 ** 31 - 2
    size = ctypes.c_size_t(0)
    assert prism.lib().prism_norm_rope_workspace_bytes(prism.F32, ctypes.byref(o), ctypes.byref(size)) == prism.EINVAL
    o.start -= 1
    assert prism.lib().prism_norm_rope_workspace_bytes(prism.F32, ctypes.byref(o), ctypes.byref(size)) == prism.OK
    o.start, o.positions = 2 ** 31 - 2, ADDRESS
    assert prism.lib().prism_norm_rope_workspace_bytes(prism.F32, ctypes.byref(o), ctypes.byref(size)) == prism.OK


@pytest.mark.parametrize("bad", [dict(fast=1.0), dict(fast=0.5), dict(factor=float("inf")), dict(original_len=-4096), dict(base=0.0), dict(base=-1.0)])
def test_frequencies_that_would_not_be_numbers(prism, bad):
    kw = dict(rot_dim=8, scaling="by_turns", factor=2.0, original_len=4096)
    assert np.all(np.isfinite(prism.rope_frequencies(**kw)[0].numpy()))
    kw.update(bad)
    with pytest.raises(prism.PrismError):
        prism.rope_frequencies(**kw)
