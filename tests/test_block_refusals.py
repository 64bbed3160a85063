"""What the operators around the layer refuse, on the CPU: the checks run on the host before anything is enqueued, so made-up addresses are
enough (no call below gets as far as a launch), and the binding's own checks see CPU tensors."""
import ctypes
import math

import pytest
import torch

import paper_2605_23764_amd as moe

P = 0x7f0000000000
INVALID, SHAPE, SMALL = -1, -2, -3
NAN, INF = math.nan, math.inf


def at(i, off=0):
    return P + i * 0x1000000 + off


@pytest.fixture(scope="module")
def lib():
    return moe.load_library()


def norm_forward(lib, T=4, H=64, dtype=1, x=at(1), gamma=at(2), beta=at(3), eps=1e-5, y=at(4), mean=at(5), rstd=at(6)):
    return lib.moe_layer_norm_forward(T, H, dtype, x, gamma, beta, eps, y, mean, rstd, None)


@pytest.mark.parametrize("want,change", [
    (INVALID, dict(dtype=2)), (INVALID, dict(dtype=-1)), (SHAPE, dict(T=-1)), (SHAPE, dict(H=0)), (SHAPE, dict(H=262145)),
    (INVALID, dict(eps=-1e-9)), (INVALID, dict(eps=NAN)), (INVALID, dict(eps=INF)), (INVALID, dict(x=None)), (INVALID, dict(y=None)),
    *[(INVALID, {n: at(7, 8)}) for n in ("x", "y", "gamma", "beta", "mean", "rstd")]])
def test_layer_norm_forward(lib, want, change):
    assert norm_forward(lib, **change) == want


def norm_backward(lib, T=4, H=64, dtype=1, dy=at(1), x=at(2), gamma=at(3), mean=at(4), rstd=at(5), dres=at(6), dx=at(7), dg=at(8), db=at(9),
                  ws=at(10), size=1 << 20):
    return lib.moe_layer_norm_backward(T, H, dtype, dy, x, gamma, mean, rstd, dres, dx, dg, db, ws, size, None)


@pytest.mark.parametrize("want,change", [
    (INVALID, dict(dtype=7)), (SHAPE, dict(H=-3)), (SHAPE, dict(T=-2)), (SMALL, dict(size=4 * 2 * 64 * 4 - 1)), (INVALID, dict(ws=None)),
    *[(INVALID, {n: None}) for n in ("dy", "x", "mean", "rstd", "dx")],
    *[(INVALID, {n: at(11, 4)}) for n in ("dy", "x", "gamma", "mean", "rstd", "dres", "dx", "dg", "db", "ws")]])
def test_layer_norm_backward(lib, want, change):
    assert norm_backward(lib, **change) == want


def drop(lib, T=4, H=64, dtype=0, v=at(1), res=at(2), p=0.5, rng=at(3), out=at(4)):
    return lib.moe_dropout_add_forward(T, H, dtype, v, res, p, rng, out, None)


DROP_BAD = [(INVALID, dict(p=-0.1)), (INVALID, dict(p=1.01)), (INVALID, dict(p=NAN)), (INVALID, dict(rng=None)), (INVALID, dict(rng=at(3, 4))),
            (INVALID, dict(dtype=3)), (SHAPE, dict(T=-1)), (SHAPE, dict(H=0))]


@pytest.mark.parametrize("want,change", DROP_BAD + [(INVALID, {n: at(5, 2)}) for n in ("v", "res", "out")] +
                         [(INVALID, {n: None}) for n in ("v", "out")])
def test_dropout_add(lib, want, change):
    assert drop(lib, **change) == want
    if "res" not in change:
        a = dict(T=4, H=64, dtype=0, v=at(1), p=0.5, rng=at(3), out=at(4)) | change
        assert lib.moe_dropout_add_backward(a["T"], a["H"], a["dtype"], a["v"], a["p"], a["rng"], a["out"], None) == want


@pytest.mark.parametrize("want,change", DROP_BAD + [(INVALID, dict(eps=NAN)), (INVALID, dict(z=at(7))), (INVALID, dict(z=None)),
                                                    (INVALID, dict(v=None)), (INVALID, dict(y=None)), (INVALID, dict(gamma=at(5, 1)))])
def test_dropout_add_layer_norm_forward(lib, want, change):
    a = dict(T=4, H=64, dtype=1, v=at(1), res=at(2), p=0.5, rng=at(3), gamma=at(4), beta=at(5), eps=1e-5, z=at(6), y=at(7), mean=at(8),
             rstd=at(9)) | change
    assert lib.moe_dropout_add_layer_norm_forward(*a.values(), None) == want


@pytest.mark.parametrize("want,change", DROP_BAD + [(SMALL, dict(size=100)), (INVALID, dict(dv=at(9))), (INVALID, dict(dv=None)),
                                                    (INVALID, dict(z=None)), (INVALID, dict(dres=at(6, 8)))])
def test_dropout_add_layer_norm_backward(lib, want, change):
    a = dict(T=4, H=64, dtype=1, dy=at(1), z=at(2), gamma=at(3), mean=at(4), rstd=at(5), dres=at(6), p=0.5, rng=at(7), dz=at(9), dv=at(10),
             dg=at(11), db=at(12), ws=at(13), size=1 << 20) | change
    assert lib.moe_dropout_add_layer_norm_backward(*a.values(), None) == want


ROUTER_SHAPES = [(SHAPE, dict(T=-1)), (SHAPE, dict(E=257)), (SHAPE, dict(E=3)), (SHAPE, dict(k=0)), (SHAPE, dict(k=17, E=32))]


@pytest.mark.parametrize("want,change", ROUTER_SHAPES + [(SMALL, dict(size=1000))] +
                         [(INVALID, {n: None}) for n in ("logits", "idx", "counts", "prob", "loss", "ws")] +
                         [(INVALID, {n: at(9, 4)}) for n in ("logits", "idx", "counts", "prob", "loss", "ws")])
def test_balance(lib, want, change):
    a = dict(T=4, E=16, k=4, logits=at(1), idx=at(2), mask=at(3), coef=0.1, counts=at(4), prob=at(5), loss=at(6), ws=at(7),
             size=moe.moe_balance_workspace_bytes(4, 16)) | change
    assert lib.moe_balance_forward(*a.values(), None) == want


@pytest.mark.parametrize("want,change", ROUTER_SHAPES + [(INVALID, dict(w=None)), (INVALID, dict(dw=None))] +
                         [(INVALID, {n: None}) for n in ("logits", "idx", "out")] +
                         [(INVALID, {n: at(9, 4)}) for n in ("logits", "idx", "w", "dw", "counts", "dloss", "out")])
def test_router_backward(lib, want, change):
    a = dict(T=4, E=16, k=4, logits=at(1), idx=at(2), w=at(3), dw=at(4), mask=at(5), coef=0.1, counts=at(6), dloss=at(7), out=at(8)) | change
    assert lib.moe_router_backward(*a.values(), None) == want


@pytest.mark.parametrize("want,change", [
    (INVALID, dict(dtype=5)), (SHAPE, dict(E=0)), (SHAPE, dict(E=257)), (SHAPE, dict(K=48)), (SHAPE, dict(K=0)), (SHAPE, dict(N=0)),
    (SHAPE, dict(K=524320)), *[(INVALID, {n: None}) for n in ("w", "q", "s")], *[(INVALID, {n: at(4, 8)}) for n in ("w", "q", "s")]])
def test_quantize(lib, want, change):
    a = dict(E=2, K=64, N=8, dtype=1, w=at(1), q=at(2), s=at(3)) | change
    assert lib.moe_quantize_w4(*a.values(), None) == want


@pytest.mark.parametrize("want,change,shape", [
    (SHAPE, {}, dict(H=96)), (SHAPE, {}, dict(E=300)), (SHAPE, dict(size=1 << 40), dict(H=65536, I=32768)), (INVALID, {}, dict(dtype=0)), (SMALL, dict(size=1000), {}),
    *[(INVALID, {n: None}, {}) for n in ("x", "logits", "q1", "s1", "q2", "s2", "out", "ws")],
    *[(INVALID, {n: at(12, 8)}, {}) for n in ("x", "logits", "q1", "s1", "q2", "s2", "out", "ws")]])
def test_forward_w4(lib, want, change, shape):
    dims = dict(T=4, H=64, I=64, E=8, E_local=8, expert_base=0, k=2, dtype=1) | shape
    s = moe.make_shape(*dims.values())
    a = dict(x=at(1), logits=at(2), q1=at(3), s1=at(4), q2=at(5), s2=at(6), out=at(7), saved=None, ws=at(8), size=1 << 30) | change
    assert lib.moe_ffn_forward_w4(ctypes.addressof(s), *a.values(), None) == want
    assert lib.moe_ffn_forward_w4(None, *a.values(), None) == INVALID


def test_workspace_queries(lib):
    assert moe.moe_layer_norm_workspace_bytes(0, 64) > 0
    assert moe.moe_layer_norm_workspace_bytes(100000, 64) == moe.moe_layer_norm_workspace_bytes(512, 64)
    for call in (lambda: moe.moe_layer_norm_workspace_bytes(4, 0), lambda: moe.moe_layer_norm_workspace_bytes(-1, 4),
                 lambda: moe.moe_balance_workspace_bytes(4, 257), lambda: moe.moe_balance_workspace_bytes(-1, 8)):
        with pytest.raises(moe.MoeError) as ei:
            call()
        assert ei.value.status == SHAPE
    assert lib.moe_layer_norm_workspace_bytes(4, 64, None) == INVALID and lib.moe_balance_workspace_bytes(4, 64, None) == INVALID


def test_binding_checks_shapes_types_and_places():
    """Every tensor is looked at: the wrong shape, type, layout or place never reaches the library."""
    bf, f32 = torch.bfloat16, torch.float32
    x = torch.zeros(4, 64, dtype=bf)
    for call in (lambda: moe.moe_layer_norm_forward(x, None, None, 1e-5, x), lambda: moe.moe_layer_norm_forward(x[0], None, None, 1e-5, x),
                 lambda: moe.moe_layer_norm_forward(x.half(), None, None, 1e-5, x), lambda: moe.moe_dropout_add_forward(x, None, 0.0, None, x),
                 lambda: moe.moe_dropout_add_backward(x, 0.0, None, x),
                 lambda: moe.moe_balance_forward(x[0], x, None, 0.1, x, x, x, None),
                 lambda: moe.moe_router_backward(x.to(f32), x.int(), None, None, None, 0.1, None, None, x),
                 lambda: moe.moe_quantize_w4(x, x, x), lambda: moe.moe_quantize_w4(x[None], x, x),
                 lambda: moe.moe_ffn_forward_w4(moe.make_shape(4, 64, 64, 8, 8, 0, 2, bf), x, x, x, x, x, x, x, None, None)):
        with pytest.raises(ValueError):
            call()
