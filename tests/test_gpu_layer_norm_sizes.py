"""Layer norm and dropout at sizes where launches take another form: arrays above 64 MB (past the caches), rows that workgroups walk over in
several turns, column sums of many long rows.  Rows do not depend on each other, so a call has the bits of calls on parts of its rows, which
stay below those sizes; sums over rows are checked in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2605_23764_amd as moe
from block_common import HALF, TORCH, U, backward_bounds, close, f64, norm_bounds
from oracle import block_oracle as bo
from test_gpu_layer_norm import EPS, _backward, _forward, _inputs, _rng

pytestmark = pytest.mark.gpu

# T x H x bytes > 2^26; whole vectors and short last ones, both types
LARGE = [(8200, 4104, "bf16"), (33600, 1001, "bf16"), (4100, 4096, "f32"), (16800, 1001, "f32"), (4700, 7168, "bf16"), (130000, 260, "bf16")]
LARGE_IDS = [f"{t}x{h}-{d}" for t, h, d in LARGE]


def _on_device(T, H, dtype, seed):
    """x with offsets and an outlier channel, dy, dres, v, gamma, beta."""
    g = torch.Generator("cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")
    x = normal(T, H) + 0.5 * normal(T, 1)
    x[:, 3::97] *= 8.0
    rest = [normal(T, H).to(TORCH[dtype]) for _ in range(3)]
    return x.to(TORCH[dtype]), *rest, (1 + 0.3 * normal(H)).to(TORCH[dtype]), (0.2 * normal(H)).to(TORCH[dtype])


def _parts(T, H, dtype):
    """Row ranges below 16 MB that start at multiples of 16 bytes."""
    step = max(8, (1 << 24) // (H * (2 if dtype == "bf16" else 4)) // 8 * 8)
    return [slice(i, min(i + step, T)) for i in range(0, T, step)]


def _factor(rows, H, p, seed, offset):
    """The oracle's mask and scale of some rows."""
    t, h = np.meshgrid(rows, np.arange(H), indexing="ij")
    thr = int(round(float(np.float32(p)) * 65536))
    words = bo.philox4x32_10([h // 8, t, np.full_like(t, offset % 2 ** 32), np.full_like(t, offset >> 32)], [seed % 2 ** 32, seed >> 32])
    word = np.choose((h % 8) // 2, words)
    bits = np.where(h % 2 == 0, word & np.uint64(0xFFFF), word >> np.uint64(16)).astype(np.int64)
    return np.where(bits >= thr, 65536.0 / (65536 - thr), 0.0)


def _sums(dy, x, mean, rstd, T, dtype):
    """dgamma and dbeta in 64 bits and their bounds, as backward_bounds has them."""
    d, xd, m, r = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    xh = (xd - m) * r
    e_xh = 2 * U * (r * (xd - m).abs() + xh.abs())
    n = (T + 1024 + 16 + 16) * U
    dg, db = (d * xh).sum(0), d.sum(0)
    e_dg, e_db = n * (d * xh).abs().sum(0) + (d.abs() * e_xh).sum(0), n * d.abs().sum(0)
    return [f64(a) for a in (dg, db, e_dg + HALF[dtype] * (dg.abs() + e_dg), e_db + HALF[dtype] * (db.abs() + e_db))]


def test_sizes_are_above_the_line():
    assert all(T * H * (2 if d == "bf16" else 4) > 1 << 26 for T, H, d in LARGE)


@pytest.mark.parametrize("T,H,dtype", LARGE, ids=LARGE_IDS)
def test_layer_norm_past_the_caches(T, H, dtype):
    print(f"layer norm T={T} H={H} {dtype}", flush=True)
    x, dy, dres, _, gamma, beta = _on_device(T, H, dtype, T)
    y, mean, rstd = _forward(x, gamma, beta)
    dx, dg, db = _backward(dy, x, gamma, mean, rstd, dres)
    for part in _parts(T, H, dtype):
        yp, mp, rp = _forward(x[part], gamma, beta)
        assert torch.equal(y[part], yp) and torch.equal(mean[part], mp) and torch.equal(rstd[part], rp), part
        assert torch.equal(dx[part], _backward(dy[part], x[part], gamma, mp, rp, dres[part], dg=False, db=False)[0]), part
    sample = torch.tensor(sorted({0, 1, T // 3, T // 2, T - 2, T - 1}), device="cuda")
    want = norm_bounds(f64(x[sample]), f64(gamma), f64(beta), EPS, dtype)
    close(y[sample], want[0], want[3], "y")
    wx, _, _, e_x, _, _, _ = backward_bounds(f64(dy[sample]), f64(x[sample]), f64(gamma), f64(mean[sample]), f64(rstd[sample]),
                                             f64(dres[sample]), dtype)
    close(dx[sample], wx, e_x, "dx")
    wg, wb, e_g, e_b = _sums(dy, x, mean, rstd, T, dtype)
    close(dg, wg, e_g, "dgamma")
    close(db, wb, e_b, "dbeta")
    for which in ("dy", "x", "dres"):                                   # in place: the stores lie over the loads
        a = dict(dy=dy.clone(), x=x.clone(), dres=dres.clone())
        got = _backward(a["dy"], a["x"], gamma, mean, rstd, a["dres"], dx=a[which])
        assert all(torch.equal(p, q) for p, q in zip(got, (dx, dg, db))), which
    same = x.clone()
    _forward(same, gamma, beta, out=same)
    assert torch.equal(same, y)


@pytest.mark.parametrize("T,H,dtype", LARGE, ids=LARGE_IDS)
def test_dropout_past_the_caches(T, H, dtype):
    """Alone: sampled rows against the oracle's mask, whole arrays in place.  With the norm: the bits of the two calls."""
    print(f"dropout T={T} H={H} {dtype}", flush=True)
    x, dy, dres, v, gamma, beta = _on_device(T, H, dtype, T + 1)
    p, seed, offset = 0.3, 2 ** 40 + 11, 2 ** 33 + 5
    rng, nan = _rng(seed, offset), float("nan")
    z = torch.full_like(x, nan)
    moe.moe_dropout_add_forward(v, x, p, rng, z)
    rows = np.unique(np.concatenate([np.arange(40), np.arange(T // 2, T // 2 + 40), np.arange(T - 40, T)]))
    at = torch.from_numpy(rows).cuda()
    f = _factor(rows, H, p, seed, offset)
    V, X = f64(v[at]), f64(x[at])
    want = X + V * f
    close(z[at], want, HALF[dtype] * np.abs(want) * (1 + 4 * U) + 2 * U * (np.abs(V * f) + np.abs(X)), "z")
    kept = z != x                                                       # what is dropped leaves the residual alone
    assert 0.6 < kept.float().mean().item() < 0.75
    for over in ("v", "x"):
        a = dict(v=v.clone(), x=x.clone())
        moe.moe_dropout_add_forward(a["v"], a["x"], p, rng, a[over])
        assert torch.equal(a[over], z), over
    dv = torch.full_like(x, nan)
    moe.moe_dropout_add_backward(dy, p, rng, dv)
    close(dv[at], f64(dy[at]) * f, (HALF[dtype] + 2 * U) * np.abs(f64(dy[at]) * f), "dv alone")
    over = dy.clone()
    moe.moe_dropout_add_backward(over, p, rng, over)
    assert torch.equal(over, dv)

    z2, y2 = torch.full_like(x, nan), torch.full_like(x, nan)
    m2, r2 = (torch.full((T,), nan, device="cuda") for _ in range(2))
    moe.moe_dropout_add_layer_norm_forward(v, x, p, rng, gamma, beta, EPS, z2, y2, m2, r2)
    y, mean, rstd = _forward(z, gamma, beta)
    assert torch.equal(z2, z) and torch.equal(y2, y) and torch.equal(m2, mean) and torch.equal(r2, rstd)
    a = dict(v=v.clone(), x=x.clone())
    moe.moe_dropout_add_layer_norm_forward(a["v"], a["x"], p, rng, gamma, beta, EPS, a["v"], a["x"], m2, r2)
    assert torch.equal(a["v"], z) and torch.equal(a["x"], y)

    ws = moe.alloc_layer_norm_workspace(T, H)
    dz, dv = torch.full_like(x, nan), torch.full_like(x, nan)
    dg, db, dg2, db2 = (torch.full_like(gamma, nan) for _ in range(4))
    moe.moe_dropout_add_layer_norm_backward(dy, z, gamma, mean, rstd, dres, p, rng, dz, dv, dg, db, ws)
    for part in _parts(T, H, dtype):                                    # dz does not depend on the mask
        dzp, dvp = torch.empty_like(x[part]), torch.empty_like(x[part])
        moe.moe_dropout_add_layer_norm_backward(dy[part], z[part], gamma, mean[part], rstd[part], dres[part], 0.0, None, dzp, dvp, None, None, None)
        assert torch.equal(dz[part], dzp) and torch.equal(dzp, dvp), part
    wg, wb, e_g, e_b = _sums(dy, z, mean, rstd, T, dtype)
    close(dg, wg, e_g, "dgamma")
    close(db, wb, e_b, "dbeta")
    wz, _, _, e_z, _, _, e_raw = backward_bounds(f64(dy[at]), f64(z[at]), f64(gamma), f64(mean[at]), f64(rstd[at]), f64(dres[at]), dtype)
    close(dz[at], wz, e_z, "dz")
    close(dv[at], wz * f, f * e_raw + (HALF[dtype] + 2 * U) * (np.abs(wz) + e_raw) * f, "dv")
    a = dict(dy=dy.clone(), z=z.clone())
    moe.moe_dropout_add_layer_norm_backward(a["dy"], a["z"], gamma, mean, rstd, dres, p, rng, a["z"], a["dy"], dg2, db2, ws)
    assert torch.equal(a["z"], dz) and torch.equal(a["dy"], dv) and torch.equal(dg2, dg) and torch.equal(db2, db)


# A launch of the forward has room for 24 rows of 520 .. 1024 elements per CU (256 of them), 12 of 2048, 8 of 2051, 3 of 7168: one to three turns
# more, the last one short; with short last vectors and in fp32.
@pytest.mark.parametrize("T,H,dtype", [(6151, 520, "bf16"), (13001, 1001, "bf16"), (12300, 1001, "f32"), (3100, 2048, "bf16"), (4200, 2051, "bf16"),
                                       (2050, 2051, "f32"), (1700, 7167, "bf16"), (24600, 65, "bf16"), (50000, 7, "f32")])
def test_forward_in_several_turns(T, H, dtype):
    print(f"turns T={T} H={H} {dtype}", flush=True)
    x, gamma, beta, _, _, v = _inputs(T, H, dtype, H + T)
    y, mean, rstd = _forward(x, gamma, beta)
    want, m, s, e_y, e_m, e_s, _ = norm_bounds(f64(x), f64(gamma), f64(beta), EPS, dtype)
    close(y, want, e_y, "y")
    close(mean, m, e_m, "mean")
    close(rstd, s, e_s, "rstd")
    z, z2 = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    moe.moe_dropout_add_layer_norm_forward(v, x, 0.4, _rng(3, 4), gamma, beta, EPS, z, y, mean, rstd)
    moe.moe_dropout_add_forward(v, x, 0.4, _rng(3, 4), z2)
    y2, mean2, rstd2 = _forward(z2, gamma, beta)
    assert torch.equal(z, z2) and torch.equal(y, y2) and torch.equal(mean, mean2) and torch.equal(rstd, rstd2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H", [(65, 8200), (150, 8193), (200, 20000)])
def test_column_sums_of_long_rows(T, H, dtype):
    """More rows than the 64 shares that the column sums of long rows are made in."""
    print(f"long rows T={T} H={H} {dtype}", flush=True)
    x, gamma, beta, dy, dres, _ = _inputs(T, H, dtype, H + T)
    _, mean, rstd = _forward(x, gamma, beta)
    dx, dg, db = _backward(dy, x, gamma, mean, rstd, dres)
    wx, wg, wb, e_x, e_g, e_b, _ = backward_bounds(f64(dy), f64(x), f64(gamma), f64(mean), f64(rstd), f64(dres), dtype)
    close(dx, wx, e_x, "dx")
    close(dg, wg, e_g, "dgamma")
    close(db, wb, e_b, "dbeta")


def test_long_rows_in_several_turns():
    """More long rows than a launch has workgroups (2^20): 17 GB an array."""
    T, H = (1 << 20) + 5, 8200
    print(f"long rows T={T} H={H}", flush=True)
    g = torch.Generator("cuda").manual_seed(1)
    x = torch.randn(T, H, generator=g, device="cuda", dtype=torch.bfloat16)
    gamma, beta = ((1 + 0.2 * torch.randn(H, generator=g, device="cuda")).to(torch.bfloat16) for _ in range(2))
    y, mean, rstd = _forward(x, gamma, beta)
    dx, _, _ = _backward(y, x, gamma, mean, rstd, None, dg=False, db=False)
    for part in [slice(i, min(i + (1 << 16), T)) for i in range(0, T, 1 << 16)]:
        yp, mp, rp = _forward(x[part], gamma, beta)
        assert torch.equal(y[part], yp) and torch.equal(mean[part], mp) and torch.equal(rstd[part], rp), part
        assert torch.equal(dx[part], _backward(yp, x[part], gamma, mp, rp, None, dg=False, db=False)[0]), part
