"""Plain fp64 CPU definitions of the routing by scores with its backward and balance bias, and of the orthogonal update.  TEST
INFRASTRUCTURE ONLY, like the rest of this package: no code, table or helper is shared with the HIP path.

Pins (tests/test_oracle_router.py): worked examples, central differences for the gradient, singular values for the update.
"""
from __future__ import annotations

import numpy as np

USUAL = (3.4445, -4.7750, 2.0315)


def scores(logits, kind):
    """[T, E]; NaN counts as -inf; -inf has score 0, several +inf share a softmax."""
    l = np.where(np.isnan(logits), -np.inf, np.asarray(logits, dtype=np.float64))
    if kind == "sigmoid":
        with np.errstate(over="ignore"):
            return 1.0 / (1.0 + np.exp(-l))
    out = np.zeros_like(l)
    for t, row in enumerate(l):
        m = row.max()
        if m == -np.inf:
            continue
        e = (row == np.inf).astype(float) if m == np.inf else np.exp(row - m)
        out[t] = e / e.sum()
    return out


def select(logits, kind, k, bias=None, n_group=1, topk_group=1):
    """(topk_idx [T, k], scores [T, E]): slot by slot, the first of the largest keys that are left."""
    s = scores(logits, kind)
    dead = np.isnan(logits) | (logits == -np.inf)
    with np.errstate(invalid="ignore"):
        key = s + (0.0 if bias is None else np.asarray(bias, dtype=np.float64))
    key[dead | np.isnan(key)] = -np.inf
    T, E = key.shape
    per = E // n_group
    idx = np.empty((T, k), dtype=np.int64)
    for t in range(T):
        value = []
        for g in range(n_group):
            two = np.sort(key[t, g * per:(g + 1) * per])[::-1][:2]
            value.append(two[0] + (two[1] if len(two) == 2 and two[1] > -np.inf else 0.0))
        stay = sorted(range(n_group), key=lambda g: (-value[g], g))[:topk_group]
        left = [e for e in range(E) if e // per in stay]
        for j in range(k):
            best = max(left, key=lambda e: (key[t, e], -e))
            idx[t, j] = best
            left.remove(best)
    return idx, s


def weights(s, idx, renormalize, scale):
    w = np.take_along_axis(s, idx, 1)
    if renormalize:
        total = w.sum(1, keepdims=True)
        w = np.divide(w, total, out=np.zeros_like(w), where=total > 0)
    return scale * w


def weights_backward(logits, kind, idx, dw, renormalize, scale):
    """Gradient of the logits by the chain rule, step by step; selected ids outside 0 .. E-1 (negative or too large) have no part."""
    s = scores(logits, kind)
    T, E = s.shape
    d = np.zeros((T, E))
    for t in range(T):
        ds = np.zeros(E)
        on = [j for j in range(idx.shape[1]) if 0 <= idx[t, j] < E]
        sel = np.array([s[t, idx[t, j]] for j in on])
        g = np.array([dw[t, j] for j in on], dtype=np.float64)
        total = sel.sum()
        if renormalize:
            part = scale * (g / total - (g * sel).sum() / total ** 2) if total > 0 else np.zeros(len(on))
        else:
            part = scale * g
        for j, v in zip(on, part):
            ds[idx[t, j]] += v
        if kind == "sigmoid":
            with np.errstate(over="ignore"):
                d[t] = ds * s[t] / (1.0 + np.exp(np.where(np.isnan(logits[t]), -np.inf, logits[t])))
        else:
            d[t] = s[t] * (ds - (ds * s[t]).sum())
    return d


def bias_step(bias, counts, rate):
    """Signs from whole numbers of any size."""
    total = sum(int(c) for c in counts)
    sign = np.array([(total > len(counts) * int(c)) - (total < len(counts) * int(c)) for c in counts], dtype=np.float64)
    return np.asarray(bias, dtype=np.float64) + rate * sign


def orthogonalize(u, steps=5, coefs=None, eps=1e-7):
    """One matrix, the polynomial of X itself."""
    x = np.asarray(u, dtype=np.float64)
    x = x / (np.sqrt((x * x).sum()) + eps)
    for i in range(steps):
        a, b, c = USUAL if coefs is None else coefs[i]
        if x.shape[0] <= x.shape[1]:
            q = x @ x.T
            x = a * x + (b * q + c * (q @ q)) @ x
        else:
            q = x.T @ x
            x = a * x + x @ (b * q + c * (q @ q))
    return x


def muon_step(g, m, w, lr, mu, nesterov, weight_decay, scale, **how):
    """(m', w') of one matrix."""
    m = mu * m + g
    o = orthogonalize(g + mu * m if nesterov else m, **how)
    return m, (1.0 - lr * weight_decay) * w - lr * scale * o
