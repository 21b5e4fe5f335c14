"""Oracle of the operators at the ends of a model: embedding, norm of the residual stream, log-probabilities and policy losses, with their gradients, written
from the definitions in fp64 numpy."""
import numpy as np


# ---- embedding

def embedding(tokens, table, scale):
    """[len(tokens), width]; a token that is no row gives zeros."""
    out = np.zeros((len(tokens), table.shape[1]))
    for i, t in enumerate(tokens):
        if 0 <= t < len(table):
            out[i] = scale * table[t]
    return out


def embedding_gradient(dout, tokens, rows, scale):
    """(the gradient, the sum of the terms' magnitudes, how many terms each row has)."""
    d, size, count = np.zeros((rows, dout.shape[1])), np.zeros((rows, dout.shape[1])), np.zeros(rows, dtype=int)
    for i, t in enumerate(tokens):
        if 0 <= t < rows:
            d[t] += scale * dout[i]
            size[t] += abs(scale) * np.abs(dout[i])
            count[t] += 1
    return d, size, count


# ---- norm

def layer_norm(h, w, b, center, eps):
    """(y, n, mean, r): n the rows before weight and bias."""
    mean = h.mean(1, keepdims=True) if center else np.zeros((len(h), 1))
    r = 1.0 / np.sqrt(((h - mean) ** 2).mean(1, keepdims=True) + eps)
    n = (h - mean) * r
    return n * w + b, n, mean, r


def layer_norm_gradient(dy, h, w, center, eps):
    """(dh, dw, db)."""
    _, n, _, r = layer_norm(h, w, np.zeros_like(w), center, eps)
    g = dy * w
    dh = g - n * (g * n).mean(1, keepdims=True)
    if center:
        dh = dh - g.mean(1, keepdims=True)
    return r * dh, (dy * n).sum(0), dy.sum(0)


# ---- log-probabilities and losses

def logprob(z, tokens, scale):
    """(logp, lse, p): 0 and rows of zeros where the token is not in the vocabulary; a row without a finite logit has p = 0."""
    n, v = z.shape
    logp, lse, p = np.zeros(n), np.zeros(n), np.zeros((n, v))
    for i, t in enumerate(tokens):
        if not 0 <= t < v:
            continue
        a = scale * z[i]
        top = a.max()
        e = np.exp(a - (0.0 if np.isneginf(top) else top))
        total = e.sum()
        with np.errstate(divide="ignore"):
            lse[i] = top + np.log(total) if total else -np.inf
        p[i] = e / total if total else 0.0
        logp[i] = -np.inf if np.isneginf(a[t]) else (a[t] - top) - np.log(total)         # (not from lse: next to a top of 1e38 the logarithm is lost)
    return logp, lse, p


def logprob_gradient(d, p, tokens, scale):
    """scale d ([j = t] - p); zeros where the token is not in the vocabulary."""
    out = np.zeros_like(p)
    for i, t in enumerate(tokens):
        if 0 <= t < p.shape[1]:
            out[i] = -p[i]
            out[i, t] += 1.0
            out[i] *= scale * d[i]
    return out


def policy_rows(logp, there, advantages=None, old=None, ref=None, weights=None, low=0.2, high=0.2, kl=0.0):
    """(weighted losses, their derivatives by logp, the magnitudes of the derivatives' derivatives) of the rows that are there."""
    n = len(logp)
    l, d, dd = np.zeros(n), np.zeros(n), np.zeros(n)
    count = int(there.sum())
    for i in range(n):
        w = (weights[i] if weights is not None else 1.0 / count) if there[i] else 0.0
        if w == 0.0:
            continue
        A = 1.0 if advantages is None else advantages[i]
        if old is None:
            l[i], d[i] = -A * logp[i], -A
        else:
            r = np.exp(logp[i] - old[i])
            held = min(max(r, 1.0 - low), 1.0 + high)
            l[i] = -min(r * A, held * A)
            d[i] = -r * A if r * A <= held * A else 0.0
            dd[i] = abs(r * A)
        if kl:
            f = ref[i] - logp[i]
            l[i] += kl * (np.exp(f) - f - 1.0)
            d[i] += kl * (1.0 - np.exp(f))
            dd[i] += kl * np.exp(f)
        l[i], d[i], dd[i] = w * l[i], w * d[i], abs(w) * dd[i]
    return l, d, dd


def logprob_apart(z, tokens, scale):
    """(logp, 1 - p of the token, p of all) with the token's own term apart from the others', so that a token next to certain keeps its digits; 0 where the token is not in the vocabulary.  Rows
    have a finite logit at the token."""
    n, v = z.shape
    logp, rest, p = np.zeros(n), np.zeros(n), np.zeros((n, v))
    for i, t in enumerate(tokens):
        if not 0 <= t < v:
            continue
        a = scale * z[i]
        e = np.exp(a - a[t])                               # odds against the token, one by one
        e[t] = 0.0
        odds = e.sum()
        logp[i], rest[i] = -np.log1p(odds), odds / (1.0 + odds)
        e[t] = 1.0
        p[i] = e / (1.0 + odds)
    return logp, rest, p
