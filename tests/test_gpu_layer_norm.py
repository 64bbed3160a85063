"""Layer norm, dropout with residual, and the two in one pass on the GPU, against the fp64 oracle: rows of every form (a few lanes, a wave,
several waves, longer than the registers), odd lengths, both types, missing optional arrays, in place, other streams, graphs."""
import numpy as np
import pytest
import torch

import paper_2605_23764_amd as moe
from block_common import HALF, TORCH, U, backward_bounds, close, f64, hidden, norm_bounds, tensor
from oracle import block_oracle as bo

pytestmark = pytest.mark.gpu

EPS = 1e-5
# lanes per row 8, 16, 32, 64; 2, 4, 14 waves; short last vectors; longer than 8192; one element
SHAPES = [(1, 1), (3, 7), (1, 64), (5, 65), (33, 130), (70, 333), (129, 512), (40, 513), (300, 1001), (17, 2048), (9, 7168), (3, 8191),
          (2, 8192), (5, 8193), (3, 20000)]
IDS = [f"{t}x{h}" for t, h in SHAPES]


def _inputs(T, H, dtype, seed, affine=True):
    r = np.random.default_rng(seed)
    x = hidden(r, T, H, dtype)
    gamma, beta = (tensor(1 + 0.3 * r.normal(size=H), dtype), tensor(0.2 * r.normal(size=H), dtype)) if affine else (None, None)
    rest = [tensor(r.normal(size=(T, H)), dtype) for _ in range(3)]
    return x, gamma, beta, *rest


def _forward(x, gamma, beta, stats=True, out=None):
    T, H = x.shape
    y = torch.full_like(x, float("nan")) if out is None else out
    mean, rstd = (torch.full((T,), float("nan"), device="cuda") for _ in range(2)) if stats else (None, None)
    moe.moe_layer_norm_forward(x, gamma, beta, EPS, y, mean, rstd)
    return y, mean, rstd


def _backward(dy, x, gamma, mean, rstd, dres, dx=None, dg=True, db=True):
    T, H = x.shape
    nan = float("nan")
    dx = torch.full_like(x, nan) if dx is None else dx
    dgamma = torch.full((H,), nan, dtype=x.dtype, device="cuda") if dg else None
    dbeta = torch.full((H,), nan, dtype=x.dtype, device="cuda") if db else None
    ws = moe.alloc_layer_norm_workspace(T, H)
    moe.moe_layer_norm_backward(dy, x, gamma, mean, rstd, dres, dx, dgamma, dbeta, ws if dg or db else None)
    return dx, dgamma, dbeta


def _opt(t):
    return None if t is None else f64(t)


@pytest.mark.parametrize("affine", [True, False], ids=["affine", "plain"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H", SHAPES, ids=IDS)
def test_layer_norm_forward_and_backward(T, H, dtype, affine):
    print(f"layer norm T={T} H={H} {dtype} affine={affine}", flush=True)
    x, gamma, beta, dy, dres, _ = _inputs(T, H, dtype, 11 * H + T, affine)
    y, mean, rstd = _forward(x, gamma, beta)
    want, m, s, e_y, e_m, e_s, _ = norm_bounds(f64(x), _opt(gamma), _opt(beta), EPS, dtype)
    close(y, want, e_y, "y")
    close(mean, m, e_m, "mean")
    close(rstd, s, e_s, "rstd")
    for with_res in (True, False):
        dx, dg, db = _backward(dy, x, gamma, mean, rstd, dres if with_res else None)
        wx, wg, wb, e_x, e_g, e_b, _ = backward_bounds(f64(dy), f64(x), _opt(gamma), f64(mean), f64(rstd),
                                                       f64(dres) if with_res else None, dtype)
        close(dx, wx, e_x, "dx")
        close(dg, wg, e_g, "dgamma")
        close(db, wb, e_b, "dbeta")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H", [(1000, 96), (2100, 520), (600, 2048), (700, 7168)])
def test_many_rows(T, H, dtype):
    """More rows than the workgroups have in hand at a time: several turns, rows past the end in the last."""
    print(f"layer norm T={T} H={H} {dtype}", flush=True)
    x, gamma, beta, dy, dres, _ = _inputs(T, H, dtype, H + T)
    y, mean, rstd = _forward(x, gamma, beta)
    close(y, *[v for i, v in enumerate(norm_bounds(f64(x), f64(gamma), f64(beta), EPS, dtype)) if i in (0, 3)], "y")
    dx, dg, db = _backward(dy, x, gamma, mean, rstd, dres)
    wx, wg, wb, e_x, e_g, e_b, _ = backward_bounds(f64(dy), f64(x), f64(gamma), f64(mean), f64(rstd), f64(dres), dtype)
    close(dx, wx, e_x, "dx")
    close(dg, wg, e_g, "dgamma")
    close(db, wb, e_b, "dbeta")
    again = _backward(dy, x, gamma, mean, rstd, dres)
    assert all(torch.equal(a, b) for a, b in zip((dx, dg, db), again))      # a fixed order of every sum


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H", [(1, 8), (1024, 64), (1025, 64), (1030, 7), (1100, 333), (1024, 1001), (1500, 1001), (384, 4096), (768, 4096),
                                 (769, 4096), (200, 8191)])
def test_backward_of_few_and_many_rows(T, H, dtype):
    """Around the limits of the backward in one launch (1024 rows, 6 MB), alone and with dropout; with one of the two sums; dx over dy."""
    print(f"few rows T={T} H={H} {dtype}", flush=True)
    x, gamma, beta, dy, dres, _ = _inputs(T, H, dtype, 3 * H + T)
    _, mean, rstd = _forward(x, gamma, beta)
    want = backward_bounds(f64(dy), f64(x), f64(gamma), f64(mean), f64(rstd), f64(dres), dtype)
    full = _backward(dy, x, gamma, mean, rstd, dres)
    for i, name in enumerate(("dx", "dgamma", "dbeta")):
        close(full[i], want[i], want[i + 3], name)
    assert torch.equal(_backward(dy, x, gamma, mean, rstd, dres, dg=False)[2], full[2])
    assert torch.equal(_backward(dy, x, gamma, mean, rstd, dres, db=False)[1], full[1])
    over = dy.clone()
    assert all(torch.equal(a, b) for a, b in zip(_backward(over, x, gamma, mean, rstd, dres, dx=over), full))
    dz, dv = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    dg, db = torch.full_like(gamma, float("nan")), torch.full_like(gamma, float("nan"))
    moe.moe_dropout_add_layer_norm_backward(dy, x, gamma, mean, rstd, dres, 0.3, _rng(5, 6), dz, dv, dg, db,
                                            moe.alloc_layer_norm_workspace(T, H))
    for got, i, name in ((dz, 0, "dz"), (dg, 1, "dgamma"), (db, 2, "dbeta")):
        close(got, want[i], want[i + 3], name)
    f = bo.dropout_factor(T, H, 0.3, 5, 6)
    close(dv, want[0] * f, f * want[6] + (HALF[dtype] + 2 * U) * (np.abs(want[0]) + want[6]) * f, "dv")


@pytest.mark.parametrize("T,H", [(30000, 72), (5300, 520), (5200, 1001), (3000, 2048), (1601, 7168)])
def test_forward_walks_rows(T, H):
    """More rows than a launch has workgroups for: several turns in the forward too, alone and with dropout."""
    print(f"walk T={T} H={H}", flush=True)
    x, gamma, beta, _, _, v = _inputs(T, H, "bf16", H + T)
    y, mean, rstd = _forward(x, gamma, beta)
    want, m, s, e_y, e_m, e_s, _ = norm_bounds(f64(x), f64(gamma), f64(beta), EPS, "bf16")
    close(y, want, e_y, "y")
    close(mean, m, e_m, "mean")
    close(rstd, s, e_s, "rstd")
    rng, z, z2 = _rng(3, 4), torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    moe.moe_dropout_add_layer_norm_forward(v, x, 0.4, rng, gamma, beta, EPS, z, y, mean, rstd)
    moe.moe_dropout_add_forward(v, x, 0.4, rng, z2)
    y2, mean2, rstd2 = _forward(z2, gamma, beta)
    assert torch.equal(z, z2) and torch.equal(y, y2) and torch.equal(mean, mean2) and torch.equal(rstd, rstd2)


def test_gradient_against_differences():
    """Central differences of the oracle's forward, in 64 bits (they are good to 1e-8), against the kernel's fp32 gradient."""
    T, H = 3, 21
    x, gamma, beta, dy, _, _ = _inputs(T, H, "f32", 77)
    _, mean, rstd = _forward(x, gamma, beta)
    dx, dg, db = _backward(dy, x, gamma, mean, rstd, None)
    X, G, B, D = f64(x), f64(gamma), f64(beta), f64(dy)
    _, _, _, e_x, e_g, e_b, _ = backward_bounds(D, X, G, *bo.layer_norm(X, G, B, EPS)[1:], None, "f32")
    _, _, _, _, e_mean, e_rstd, e_xh = norm_bounds(X, G, B, EPS, "f32")
    slack = np.abs(D * G).sum(axis=1, keepdims=True) * (e_rstd + e_mean)[:, None] * 4 + 1e-7   # mean and rstd are the kernel's own
    h = 1e-6

    def diff(a, fn):
        out = np.zeros_like(a)
        for i in np.ndindex(a.shape):
            p, q = a.copy(), a.copy()
            p[i] += h
            q[i] -= h
            out[i] = (fn(p) - fn(q)) / (2 * h)
        return out
    close(dx, diff(X, lambda a: (D * bo.layer_norm(a, G, B, EPS)[0]).sum()), e_x + slack, "dx")
    close(dg, diff(G, lambda a: (D * bo.layer_norm(X, a, B, EPS)[0]).sum()), e_g + (np.abs(D) * e_xh).sum(axis=0) + 1e-7, "dgamma")
    close(db, diff(B, lambda a: (D * bo.layer_norm(X, G, a, EPS)[0]).sum()), e_b + 1e-7, "dbeta")


@pytest.mark.parametrize("H", [72, 1001, 9001])
def test_optional_outputs_and_in_place(H):
    T = 13
    x, gamma, beta, dy, dres, _ = _inputs(T, H, "bf16", H)
    y, mean, rstd = _forward(x, gamma, beta)
    assert torch.equal(_forward(x, gamma, beta, stats=False)[0], y)
    same = x.clone()
    _forward(same, gamma, beta, out=same)
    assert torch.equal(same, y)
    full = _backward(dy, x, gamma, mean, rstd, dres)
    assert torch.equal(_backward(dy, x, gamma, mean, rstd, dres, dg=False, db=False)[0], full[0])
    part = _backward(dy, x, gamma, mean, rstd, dres, dg=False)
    assert torch.equal(part[0], full[0]) and torch.equal(part[2], full[2])
    part = _backward(dy, x, gamma, mean, rstd, dres, db=False)
    assert torch.equal(part[1], full[1])
    for which in ("dy", "x", "dres"):
        a = dict(dy=dy.clone(), x=x.clone(), dres=dres.clone())
        got = _backward(a["dy"], a["x"], gamma, mean, rstd, a["dres"], dx=a[which])
        assert all(torch.equal(p, q) for p, q in zip(got, full)), which


def test_rows_do_not_meet():
    """A row of NaN, one of infinities and one of zeros: the others keep their bits; a constant row has y = beta."""
    x, gamma, beta, dy, dres, _ = _inputs(12, 200, "bf16", 5)
    y, mean, rstd = _forward(x, gamma, beta)
    odd = x.clone()
    odd[2], odd[5, 7], odd[8], odd[9] = float("nan"), float("inf"), 0.0, 3.5
    yo, mo, ro = _forward(odd, gamma, beta)
    keep = [0, 1, 3, 4, 6, 7, 10, 11]
    assert torch.equal(yo[keep], y[keep]) and torch.equal(mo[keep], mean[keep])
    assert torch.isnan(yo[2].float()).all() and torch.isnan(yo[5].float()).all()
    assert torch.equal(yo[8], beta) and torch.equal(yo[9], beta)
    dx, _, _ = _backward(dy, x, gamma, mean, rstd, dres)
    dxo, _, _ = _backward(dy, odd, gamma, mo, ro, dres)
    assert torch.equal(dxo[keep], dx[keep])


def test_nothing_to_do():
    x = torch.empty(0, 256, dtype=torch.bfloat16, device="cuda")
    e = torch.empty(0, device="cuda")
    g = torch.ones(256, dtype=torch.bfloat16, device="cuda")
    moe.moe_layer_norm_forward(x, g, g, EPS, x, e, e)
    _, dg, db = _backward(x, x, g, e, e, None)
    assert (dg == 0).all() and (db == 0).all()
    moe.moe_dropout_add_forward(x, x, 0.5, torch.zeros(2, dtype=torch.int64, device="cuda"), x)


# ---- dropout ----
def _rng(seed, offset):
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H", SHAPES + [(2000, 40), (257, 4104)], ids=IDS + ["2000x40", "257x4104"])
def test_dropout_add(T, H, dtype):
    print(f"dropout T={T} H={H} {dtype}", flush=True)
    r = np.random.default_rng(H + 3 * T)
    v, res = (tensor(r.normal(size=(T, H)), dtype) for _ in range(2))
    for p, seed, offset in ((0.1, 2 ** 40 + 5, 2 ** 33 + 1), (0.5, -3, 7), (1.0, 1, 1)):
        f = bo.dropout_factor(T, H, p, seed, offset)
        rng = _rng(seed, offset)
        out = torch.full_like(v, float("nan"))
        moe.moe_dropout_add_forward(v, res, p, rng, out)
        want = f64(res) + f64(v) * f
        close(out, want, HALF[dtype] * np.abs(want) * (1 + 4 * U) + 2 * U * (np.abs(f64(v) * f) + np.abs(f64(res))), "out")
        assert torch.equal(out[torch.from_numpy(f == 0).cuda()], res[torch.from_numpy(f == 0).cuda()])
        # what is dropped may hold anything
        wild = v.clone()
        wild[torch.from_numpy(f == 0).cuda()] = float("nan")
        again = torch.empty_like(out)
        moe.moe_dropout_add_forward(wild, res, p, rng, again)
        assert torch.equal(again, out)
        alone, dv = torch.full_like(v, float("nan")), torch.full_like(v, float("nan"))
        moe.moe_dropout_add_forward(v, None, p, rng, alone)
        moe.moe_dropout_add_backward(v, p, rng, dv)
        want = f64(v) * f
        close(dv, want, (HALF[dtype] + 2 * U) * np.abs(want), "dv")        # nothing but 0 where it is dropped
        assert torch.equal(dv, alone)
        moe.moe_dropout_add_forward(again, res, p, rng, again)             # in place
        moe.moe_dropout_add_forward(out, res, p, rng, out)
        assert torch.equal(out, again)


def test_no_dropout_needs_no_generator():
    v, res = (torch.randn(5, 100, device="cuda") for _ in range(2))
    out = torch.empty_like(v)
    moe.moe_dropout_add_forward(v, res, 0.0, None, out)
    assert torch.equal(out, v + res)
    moe.moe_dropout_add_backward(v, 0.0, None, out)
    assert torch.equal(out, v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H", SHAPES, ids=IDS)
def test_dropout_add_layer_norm(T, H, dtype):
    """Forward: the bits of the two calls.  Backward: the oracle on the z that the forward stored."""
    print(f"dropout + norm T={T} H={H} {dtype}", flush=True)
    x, gamma, beta, dy, dres, v = _inputs(T, H, dtype, 7 * H + T)
    nan = float("nan")
    for p, res in ((0.3, x), (0.0, x), (0.3, None)):
        rng = _rng(42 + H, 1000) if p else None
        z, y = torch.full_like(x, nan), torch.full_like(x, nan)
        mean, rstd = (torch.full((T,), nan, device="cuda") for _ in range(2))
        moe.moe_dropout_add_layer_norm_forward(v, res, p, rng, gamma, beta, EPS, z, y, mean, rstd)
        z2 = torch.full_like(x, nan)
        moe.moe_dropout_add_forward(v, res, p, rng, z2)
        y2, mean2, rstd2 = _forward(z2, gamma, beta)
        assert torch.equal(z, z2) and torch.equal(y, y2) and torch.equal(mean, mean2) and torch.equal(rstd, rstd2)
        dz, dv = torch.full_like(x, nan), torch.full_like(x, nan)
        dg, db = torch.full_like(gamma, nan), torch.full_like(gamma, nan)
        moe.moe_dropout_add_layer_norm_backward(dy, z, gamma, mean, rstd, dres, p, rng, dz, dv, dg, db, moe.alloc_layer_norm_workspace(T, H))
        wz, wg, wb, e_z, e_g, e_b, e_raw = backward_bounds(f64(dy), f64(z), f64(gamma), f64(mean), f64(rstd), f64(dres), dtype)
        close(dz, wz, e_z, "dz")
        close(dg, wg, e_g, "dgamma")
        close(db, wb, e_b, "dbeta")
        f = bo.dropout_factor(T, H, p, 42 + H, 1000)
        close(dv, wz * f, f * e_raw + (HALF[dtype] + 2 * U) * (np.abs(wz) + e_raw) * f, "dv")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H", [(9, 61), (40, 520), (300, 1001), (5, 4099), (3, 9001)])
def test_dropout_add_layer_norm_in_place(T, H, dtype):
    """Every output over an input of its shape: the same bits (short last vectors read past neighbours that are being written)."""
    x, gamma, beta, dy, dres, v = _inputs(T, H, dtype, H)
    rng, p = _rng(7, 8), 0.3
    stats = [torch.empty(T, device="cuda") for _ in range(2)]
    z, y = torch.empty_like(x), torch.empty_like(x)
    moe.moe_dropout_add_layer_norm_forward(v, x, p, rng, gamma, beta, EPS, z, y, *stats)
    for zi, yi in (("v", "x"), ("x", "v"), ("x", None), (None, "v")):
        a = dict(v=v.clone(), x=x.clone())
        zo, yo = (a[n] if n else torch.empty_like(x) for n in (zi, yi))
        moe.moe_dropout_add_layer_norm_forward(a["v"], a["x"], p, rng, gamma, beta, EPS, zo, yo, *(torch.empty_like(s) for s in stats))
        assert torch.equal(zo, z) and torch.equal(yo, y), (zi, yi)
    ws, dg, db = moe.alloc_layer_norm_workspace(T, H), torch.empty_like(gamma), torch.empty_like(gamma)

    def backward(a, dz, dv):
        moe.moe_dropout_add_layer_norm_backward(a["dy"], a["z"], gamma, *stats, a["dres"], p, rng, dz, dv, dg, db, ws)
        return dz.clone(), dv.clone(), dg.clone(), db.clone()
    want = backward(dict(dy=dy, z=z, dres=dres), torch.empty_like(x), torch.empty_like(x))
    for zi, vi in (("dy", "z"), ("z", "dres"), ("dres", "dy")):
        a = dict(dy=dy.clone(), z=z.clone(), dres=dres.clone())
        assert all(torch.equal(p_, q_) for p_, q_ in zip(backward(a, a[zi], a[vi]), want)), (zi, vi)


def test_graph_replays_draw_new_masks():
    """The generator's state is read when the launch runs: replays of one captured step with a changed offset, eager work in between."""
    T, H, p = 96, 520, 0.25
    x, gamma, beta, dy, dres, v = _inputs(T, H, "bf16", 1)
    rng = _rng(9, 0)
    out = {n: torch.empty_like(x) for n in ("z", "y", "dz", "dv")}
    mean, rstd = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    dg, db, ws = torch.empty_like(gamma), torch.empty_like(gamma), moe.alloc_layer_norm_workspace(T, H)

    def step():
        moe.moe_dropout_add_layer_norm_forward(v, x, p, rng, gamma, beta, EPS, out["z"], out["y"], mean, rstd)
        moe.moe_dropout_add_layer_norm_backward(dy, out["z"], gamma, mean, rstd, dres, p, rng, out["dz"], out["dv"], dg, db, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    seen = []
    for offset in (1, 2, 1):
        rng[1] = offset
        for t in (*out.values(), mean, rstd, dg, db):
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*out.values(), mean, rstd, dg, db)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (*out.values(), mean, rstd, dg, db)))
        seen.append(got[0])
    assert torch.equal(seen[0], seen[2]) and not torch.equal(seen[0], seen[1])


def test_on_another_stream():
    x, gamma, beta, _, _, _ = _inputs(50, 300, "f32", 2)
    want, _, _ = _forward(x, gamma, beta)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    y = torch.full_like(x, float("nan"))
    torch.cuda.synchronize()
    moe.moe_layer_norm_forward(x, gamma, beta, EPS, y, stream=s)
    s.synchronize()
    assert torch.equal(y, want)
