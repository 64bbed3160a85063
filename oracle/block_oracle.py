"""Plain fp64 CPU definitions of the operators around the layer: layer norm, dropout with residual, balance loss and the router's
backward, 4-bit weights.  TEST INFRASTRUCTURE ONLY, like the rest of this package: no code, table or helper is shared with the HIP path.

Pins (tests/test_oracle_block.py): published known answers of the generator, central differences for every gradient, brute force for the
4-bit codes.
"""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def philox4x32_10(counter, key):
    """Philox4x32 with ten rounds (Salmon et al., 2011).  counter: four arrays of integers below 2^32, key: two; four arrays."""
    c = [np.asarray(v, dtype=np.uint64) for v in counter]
    k = [int(v) for v in key]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & low, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def dropout_factor(T, H, p, seed, offset):
    """[T, H] of 0 (dropped) or 65536 / (65536 - thr): element (t, h) has half h % 2 of word (h % 8) / 2 of the counter
    (h / 8, t, offset) under the key seed, and is kept if those 16 bits are at least thr = 65536 p."""
    thr = int(round(float(np.float32(p)) * 65536))
    if thr == 0:
        return np.ones((T, H))
    if thr == 65536:
        return np.zeros((T, H))
    seed, offset = seed % 2 ** 64, offset % 2 ** 64
    h, t = np.meshgrid(np.arange(H), np.arange(T))
    words = philox4x32_10([h // 8, t, np.full_like(h, offset % 2 ** 32), np.full_like(h, offset >> 32)], [seed % 2 ** 32, seed >> 32])
    word = np.choose((h % 8) // 2, words)
    bits = np.where(h % 2 == 0, word & np.uint64(0xFFFF), word >> np.uint64(16)).astype(np.int64)
    return np.where(bits >= thr, 65536.0 / (65536 - thr), 0.0)


def layer_norm(x, gamma, beta, eps):
    """(y, mean, rstd); gamma, beta may be None."""
    mean = x.mean(axis=1)
    d = x - mean[:, None]
    rstd = 1.0 / np.sqrt((d * d).mean(axis=1) + eps)
    y = d * rstd[:, None]
    if gamma is not None:
        y = y * gamma
    if beta is not None:
        y = y + beta
    return y, mean, rstd


def layer_norm_backward(dy, x, gamma, mean, rstd, dres=None):
    """(dx + dres, dgamma, dbeta)."""
    xh = (x - mean[:, None]) * rstd[:, None]
    t = dy if gamma is None else dy * gamma
    dx = rstd[:, None] * (t - t.mean(axis=1, keepdims=True) - xh * (t * xh).mean(axis=1, keepdims=True))
    return dx if dres is None else dx + dres, (dy * xh).sum(axis=0), dy.sum(axis=0)


def router_probabilities(logits):
    """Softmax over all experts; rows of -inf alone are 0."""
    m = logits.max(axis=1, keepdims=True)
    empty = np.isneginf(m)
    ex = np.exp(logits - np.where(empty, 0.0, m))
    s = ex.sum(axis=1, keepdims=True)
    return np.where(empty, 0.0, ex / np.where(empty, 1.0, s))


def balance(logits, topk_idx, mask, coef):
    """(counts [E], tokens n, prob_sum [E], loss)."""
    E, k = logits.shape[1], topk_idx.shape[1]
    on = np.ones(len(logits), dtype=bool) if mask is None else np.asarray(mask) != 0
    ids = topk_idx[on].ravel()
    counts = np.bincount(ids[(ids >= 0) & (ids < E)], minlength=E)
    n = int(on.sum())
    prob_sum = router_probabilities(logits[on]).sum(axis=0)
    loss = coef * E * float((counts / (k * n)) @ (prob_sum / n)) if n else 0.0
    return counts, n, prob_sum, loss


def router_backward(logits, topk_idx, topk_w, dtopk_w, mask, coef, counts, n, dloss=1.0):
    """Gradient of the logits; topk_w and dtopk_w, or counts, may be None."""
    T, E = logits.shape
    k = topk_idx.shape[1]
    d = np.zeros((T, E))
    if counts is not None and n > 0:
        q = router_probabilities(logits)
        f = counts / (k * n)
        d = dloss * coef * E / n * q * (f - (q @ f)[:, None])
        if mask is not None:
            d[np.asarray(mask) == 0] = 0.0
    if topk_w is not None:
        g = topk_w * (dtopk_w - (topk_w * dtopk_w).sum(axis=1, keepdims=True))
        for t in range(T):
            for j in range(k):
                if 0 <= topk_idx[t, j] < E:
                    d[t, topk_idx[t, j]] += g[t, j]
    return d


def quantize_w4(w):
    """w [E, K, N] -> (q [E, K/32, N, 16] uint8, scale [E, K/32, N] uint8)."""
    E, K, N = w.shape
    v = w.astype(np.float64).reshape(E, K // 32, 32, N).transpose(0, 1, 3, 2)          # [E, G, N, 32]
    top = np.abs(v).max(axis=3)
    bad = ~np.isfinite(v).all(axis=3)
    with np.errstate(invalid="ignore", divide="ignore"):
        e = np.floor(np.log2(np.where((top > 0) & ~bad, top, 4.0))).astype(int)
    e = np.maximum(e, -126)                                                            # float32's smallest exponent
    s = np.where(top > 0, np.maximum(e - 2 + 127, 1), 127)
    m = np.abs(np.where(bad[..., None], 0.0, v)) * 2.0 ** (127 - s)[..., None]
    dist = np.abs(m[..., None] - E2M1)
    order = np.argsort(dist + 1e-9 * (np.arange(8) % 2), axis=-1, kind="stable")       # a tie goes to the even code
    code = order[..., 0] + 8 * np.where(bad[..., None], False, np.signbit(v))
    q = code[..., 0::2] | code[..., 1::2] << 4
    return q.astype(np.uint8), np.where(bad, 255, s).astype(np.uint8)


def dequantize_w4(q, scale):
    """The weights [E, K, N] that blocks stand for."""
    E, G, N, _ = q.shape
    code = np.stack([q & 15, q >> 4], axis=-1).reshape(E, G, N, 32).astype(int)
    v = np.where(code >= 8, -1.0, 1.0) * E2M1[code & 7]
    with np.errstate(over="ignore"):
        v = v * np.where(scale == 255, np.nan, 2.0 ** (scale.astype(float) - 127))[..., None]
    return v.transpose(0, 1, 3, 2).reshape(E, G * 32, N)
