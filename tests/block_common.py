"""Inputs and error bounds of the GPU tests of layer norm and dropout (operators around the layer)."""
import numpy as np
import torch

U = 2.0 ** -24                                    # fp32: half a step
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}     # one rounding to the storage type, relative
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def tensor(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(TORCH[dtype])


def f64(t):
    return t.detach().double().cpu().numpy()


def hidden(r, T, H, dtype):
    """Rows with an offset and an outlier channel, as a residual stream has them."""
    x = r.normal(size=(T, H)) + 0.5 * r.normal(size=(T, 1))
    x[:, 3::97] *= 8.0
    return tensor(x, dtype)


def chain(H):
    """Roundings on the way of one term through a row sum: a lane's own terms one after the other, 6 exchanges in the wave, 16 waves;
    and 16 for the arithmetic around it."""
    return 8 * -(-H // 8192) + 6 + 16 + 16


def close(got, want, tol, what):
    """|got - want| <= tol, element by element."""
    got = f64(got) if isinstance(got, torch.Tensor) else got
    err = np.abs(got - want)
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.max(err / np.maximum(tol, 1e-300)):.3g} of what is allowed"


def norm_bounds(x, gamma, beta, eps, dtype):
    """(y, mean, rstd, bounds of their errors, error of xh) of a layer norm computed in fp32 from the values x."""
    from oracle import block_oracle as bo
    H = x.shape[1]
    c = chain(H) * U
    y, mean, rstd = bo.layer_norm(x, gamma, beta, eps)
    xh = (x - mean[:, None]) * rstd[:, None]
    e_mean = c * np.abs(x).mean(axis=1)
    # the variance of values that are each off by e_mean and a rounding: relative 2 e rstd, and the sum's own roundings
    e_d = e_mean[:, None] + U * (np.abs(x) + np.abs(mean)[:, None])
    e_rstd = rstd * (c + (np.abs(xh) * e_d).mean(axis=1) * rstd + 4 * U)
    e_xh = rstd[:, None] * e_d + np.abs(xh) * (e_rstd / rstd)[:, None] + 2 * U * np.abs(xh)
    g = np.ones(H) if gamma is None else np.abs(gamma)
    b = np.zeros(H) if beta is None else np.abs(beta)
    e_y = e_xh * g + 2 * U * (np.abs(xh) * g + b) + HALF[dtype] * (np.abs(y) + e_xh * g)
    return y, mean, rstd, e_y, e_mean + U * np.abs(mean), e_rstd, e_xh


def backward_bounds(dy, x, gamma, mean, rstd, dres, dtype):
    """(dx, dgamma, dbeta, their bounds, bound of dx before its rounding) for the backward on fp32 mean and rstd as given."""
    from oracle import block_oracle as bo
    T, H = x.shape
    c = chain(H) * U
    dx, dg, db = bo.layer_norm_backward(dy, x, gamma, mean, rstd, dres)
    r = rstd[:, None]
    xh = (x - mean[:, None]) * r
    t = dy if gamma is None else dy * gamma
    e_xh = 2 * U * (r * np.abs(x - mean[:, None]) + np.abs(xh))
    row = lambda a: a.mean(axis=1, keepdims=True)  # noqa: E731
    m2 = np.abs(row(t * xh))
    e_m1 = c * row(np.abs(t))
    e_m2 = c * row(np.abs(t * xh)) + row(np.abs(t) * e_xh)
    e_in = U * np.abs(t) + e_m1 + np.abs(xh) * e_m2 + m2 * e_xh
    e_raw = r * (e_in + 4 * U * (np.abs(t) + row(np.abs(t)) + np.abs(xh) * m2)) + 2 * U * np.abs(dx)
    if dres is not None:
        e_raw = e_raw + U * np.abs(dres)
    # column sums: a workgroup's rows one after the other (at most T of them), its rows in hand, 16 shares of up to 256 partials
    n = (T + 1024 + 16 + 16) * U
    e_dg = n * np.abs(dy * xh).sum(axis=0) + (np.abs(dy) * e_xh).sum(axis=0)
    e_db = n * np.abs(dy).sum(axis=0)
    return dx, dg, db, e_raw + HALF[dtype] * (np.abs(dx) + e_raw), e_dg + HALF[dtype] * (np.abs(dg) + e_dg), \
        e_db + HALF[dtype] * (np.abs(db) + e_db), e_raw
