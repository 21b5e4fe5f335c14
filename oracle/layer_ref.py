"""Oracle of the operators of a transformer layer: dropout, norm and rotation of queries and keys, attention, with their gradients, written
from the definitions in fp64 numpy, one (sequence, head) at a time."""
import numpy as np

DROPOUT_TAG = 7


# ---- dropout

def philox4x32_10(counter, key):
    """Ten rounds on four uint32 arrays (Salmon et al., SC'11), in Python-width integers held as uint64."""
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    k = [int(x) for x in key]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & low, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def dropout_kept(first, count, p, seed, offset):
    """(which of the elements first .. first + count - 1 stay, what they are multiplied by)."""
    e = np.arange(first, first + count, dtype=np.uint64)
    g = e // np.uint64(8)
    w = np.stack(philox4x32_10((g & np.uint64(0xFFFFFFFF), g >> np.uint64(32), np.full_like(g, offset), np.full_like(g, DROPOUT_TAG)),
                               (seed & 0xFFFFFFFF, seed >> 32)))
    word = w[(e % np.uint64(8) // np.uint64(2)).astype(np.int64), np.arange(count)]
    u = np.where(e % np.uint64(2) == 0, word & np.uint64(0xFFFF), word >> np.uint64(16))
    limit = int(np.rint(p * 65536))
    return u >= limit, 65536.0 / (65536 - limit)


# ---- norm and rotation

def _pairs(dim, rot, interleaved):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def _turn(x, positions, inv_freq, interleaved, scale, sign):
    rot = 2 * len(inv_freq)
    a, b = _pairs(x.shape[-1], rot, interleaved)
    z = x[..., a] + 1j * x[..., b]
    angle = positions.astype(np.float64)[:, :, None, None] * np.asarray(inv_freq, dtype=np.float64)
    z = z * scale * np.exp(1j * sign * angle)
    y = x.copy()
    y[..., a], y[..., b] = z.real, z.imag
    return y


def norm_rope(x, positions, inv_freq, weight, norm, interleaved, scale, eps):
    """x [batch, token, head, dim] in fp64."""
    y = x
    if norm:
        y = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * weight
    return _turn(y, positions, inv_freq, interleaved, scale, 1.0)


def norm_rope_grad(dy, x, positions, inv_freq, weight, norm, interleaved, scale, eps):
    """(dx, dweight)."""
    dn = _turn(dy, positions, inv_freq, interleaved, scale, -1.0)
    if not norm:
        return dn, None
    r = 1.0 / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
    dh = dn * weight
    return r * (dh - x * r * r * np.mean(dh * x, axis=-1, keepdims=True)), np.sum(dn * x * r, axis=(0, 1, 2))


# ---- attention

def visible(n, m, causal=False, prefix=None, keys=None, q_doc=None, k_doc=None):
    """[n, m] of one sequence, and the distances."""
    keys = m if keys is None else min(max(int(keys), 0), m)
    at, j = np.arange(n)[:, None] + keys - n, np.arange(m)[None, :]
    see = np.broadcast_to(j < keys, (n, m)).copy()
    if causal:
        see &= (j <= at) | (j < (0 if prefix is None else int(prefix)))
    if q_doc is not None:
        see &= (np.asarray(q_doc)[:, None] == np.asarray(k_doc)[None, :]) & (np.asarray(q_doc)[:, None] >= 0)
    return see, np.abs(at - j)


def attention_head(q, k, v, see, far, scale, softcap=0.0, slope=0.0, dout=None):
    """One head: a dict with out, lse and, with dout, dq, dk, dv; and the weights p and score gradients ds that made them."""
    see_row = see.any(axis=1)
    k, v = np.where(see.any(axis=0)[:, None], k, 0.0), np.where(see.any(axis=0)[:, None], v, 0.0)
    q = np.where(see_row[:, None], q, 0.0)
    raw = scale * (q @ k.T)
    t = np.tanh(raw / softcap) if softcap else None
    a = (softcap * t if softcap else raw) - slope * far
    a = np.where(see, a, -np.inf)
    top = np.where(see_row, a.max(axis=1, initial=-np.inf), 0.0)[:, None]
    e = np.exp(a - top)
    total = e.sum(axis=1, keepdims=True)
    p = e / np.where(total == 0, 1.0, total)
    with np.errstate(divide="ignore"):
        r = {"out": p @ v, "lse": np.where(see_row, top[:, 0] + np.log(total[:, 0]), -np.inf), "p": p, "a": a}
    if dout is not None:
        dout = np.where(see_row[:, None], dout, 0.0)
        ds = p * (dout @ v.T - np.sum(dout * r["out"], axis=1, keepdims=True))
        if softcap:
            ds = ds * (1.0 - t * t)
        ds = ds * scale
        r.update(dq=ds @ k, dk=ds.T @ q, dv=p.T @ dout, ds=ds)
    return r
