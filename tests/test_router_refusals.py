"""What the routing by scores, the router's projection and the orthogonal updates refuse, on the CPU: the checks run on the host before
anything is enqueued, so made-up addresses are enough (no call below gets as far as a launch), and the binding's own checks see CPU tensors."""
import ctypes
import math

import pytest
import torch

import paper_2605_23764_amd as moe
from paper_2605_23764_amd.binding import _MoeSaved

P = 0x7f0000000000
INVALID, SHAPE, SMALL = -1, -2, -3
NAN, INF = math.nan, math.inf
HUGE = 1 << 60


def at(i, off=0):
    return P + i * 0x10000000 + off


@pytest.fixture(scope="module")
def lib():
    return moe.load_library()


# ---- routing by scores ----

SCORES = dict(score="sigmoid", n_group=4, topk_group=2, renormalize=True, scale=2.0)
BAD_SCORES = [(INVALID, dict(score=2)), (INVALID, dict(score=-1)), (INVALID, dict(scale=NAN)), (INVALID, dict(scale=INF)),
              (INVALID, dict(renormalize=2)), (SHAPE, dict(n_group=0)), (SHAPE, dict(n_group=-4)), (SHAPE, dict(n_group=3)),
              (SHAPE, dict(n_group=32)), (SHAPE, dict(topk_group=0)), (SHAPE, dict(topk_group=5)), (SHAPE, dict(n_group=8, topk_group=1))]


def route(lib, scores=None, shape=(100, 64, 64, 32, 16, 8, 5, moe.MOE_BF16), logits=at(1), bias=at(2), saved=True, ws=at(3), size=1 << 30, mode=0, **change):
    s = moe.make_shape(*shape)
    sc = moe.make_scores(**{**SCORES, **(scores or {})})
    sv = _MoeSaved(*(change.get(n, at(10 + i)) for i, (n, _) in enumerate(_MoeSaved._fields_)))
    return lib.moe_route_scores(ctypes.addressof(s), ctypes.addressof(sc) if scores is not False else None, logits, bias,
                                ctypes.addressof(sv) if saved else None, ws, size, mode, None)


@pytest.mark.parametrize("want,change", [
    *[(w, dict(scores=c)) for w, c in BAD_SCORES], (INVALID, dict(scores=False)), (INVALID, dict(mode=2)), (INVALID, dict(mode=-1)), (INVALID, dict(logits=None)), (INVALID, dict(logits=at(1, 8))),
    (INVALID, dict(bias=at(2, 4))), (INVALID, dict(saved=False)), (INVALID, dict(topk_w=None)), (INVALID, dict(row_of=at(9, 4))),
    (INVALID, dict(ws=None)), (INVALID, dict(ws=at(3, 8))), (SMALL, dict(size=16)), (SHAPE, dict(shape=(100, 64, 64, 320, 16, 8, 5, 1))),
    (SHAPE, dict(shape=(-1, 64, 64, 32, 16, 8, 5, 1))), (SHAPE, dict(shape=(100, 64, 64, 32, 16, 20, 5, 1)))])
def test_route_scores(lib, want, change):
    assert route(lib, **change) == want


def test_route_scores_of_no_tokens(lib):
    assert route(lib, shape=(0, 64, 64, 32, 16, 8, 5, 1), logits=None, ws=None, size=0, saved=False) == 0
    assert route(lib, shape=(0, 64, 64, 32, 16, 8, 5, 1), scores=dict(n_group=3)) == SHAPE


def route_backward(lib, T=10, E=32, k=5, scores=None, logits=at(1), idx=at(2), dw=at(3), dadd=at(4), out=at(5)):
    sc = moe.make_scores(**{**SCORES, **(scores or {})})
    return lib.moe_route_scores_backward(T, E, k, ctypes.addressof(sc) if scores is not False else None, logits, idx, dw, dadd, out, None)


@pytest.mark.parametrize("want,change", [
    *[(w, dict(scores=c)) for w, c in BAD_SCORES], (INVALID, dict(scores=False)), (SHAPE, dict(T=-1)), (SHAPE, dict(E=260)), (SHAPE, dict(k=17)),
    (SHAPE, dict(k=0)), *[(INVALID, {n: None}) for n in ("logits", "idx", "dw", "out")],
    *[(INVALID, {n: at(6, 4)}) for n in ("logits", "idx", "dw", "dadd", "out")]])
def test_route_scores_backward(lib, want, change):
    assert route_backward(lib, **change) == want


@pytest.mark.parametrize("want,args", [
    (SHAPE, (0, at(1), 1e-3, at(2), at(3))), (SHAPE, (257, at(1), 1e-3, at(2), at(3))), (INVALID, (8, at(1), NAN, at(2), at(3))),
    (INVALID, (8, None, 1e-3, at(2), at(3))), (INVALID, (8, at(1), 1e-3, None, at(3))), (INVALID, (8, at(1), 1e-3, at(2), None)),
    (INVALID, (8, at(1, 4), 1e-3, at(2), at(3))), (INVALID, (8, at(1), 1e-3, at(2, 8), at(3)))])
def test_bias_update(lib, want, args):
    assert lib.moe_bias_update(*args, None) == want


def combine_w4(lib, saved=True, dtype=moe.MOE_BF16, T=100, ws=at(3), size=1 << 34, **change):
    s = moe.make_shape(T, 64, 64, 32, 16, 8, 5, dtype)
    sv = _MoeSaved(*(at(20 + i) for i in range(11)))
    ptrs = [change.get(n, at(10 + i)) for i, n in enumerate(("x", "q1", "s1", "q2", "s2", "out"))]
    return lib.moe_dispatch_to_combine_w4(ctypes.addressof(s), *ptrs, ctypes.addressof(sv) if saved else None, ws, size, None)


@pytest.mark.parametrize("want,change", [
    (INVALID, dict(saved=False)), (INVALID, dict(dtype=moe.MOE_F32)), (INVALID, dict(ws=None)), (SMALL, dict(size=64)),
    *[(INVALID, {n: None}) for n in ("x", "q1", "s1", "q2", "s2", "out")], *[(INVALID, {n: at(9, 8)}) for n in ("x", "q1", "s1", "q2", "s2", "out")]])
def test_dispatch_to_combine_w4(lib, want, change):
    assert combine_w4(lib, **change) == want


# ---- the router's projection ----

def project(lib, T=10, H=96, E=24, dtype=1, x=at(1), w=at(2), logits=at(3), ws=at(4), size=1 << 30):
    return lib.moe_router_project(T, H, E, dtype, x, w, logits, ws, size, None)


def project_backward(lib, T=10, H=96, E=24, dtype=1, d=at(1), x=at(2), w=at(3), dres=at(4), dx=at(5), dw=at(6), ws=at(7), size=1 << 30):
    return lib.moe_router_project_backward(T, H, E, dtype, d, x, w, dres, dx, dw, ws, size, None)


SIZES = [(SHAPE, dict(T=-1)), (SHAPE, dict(H=0)), (SHAPE, dict(H=(1 << 18) + 1)), (SHAPE, dict(E=0)), (SHAPE, dict(E=257)), (INVALID, dict(dtype=2)),
         (SHAPE, dict(T=2 ** 31 - 1, H=1 << 18))]


@pytest.mark.parametrize("want,change", SIZES + [(INVALID, {n: None}) for n in ("x", "w", "logits", "ws")] +
                         [(INVALID, {n: at(5, 8)}) for n in ("x", "w", "logits", "ws")] + [(SMALL, dict(size=15))])
def test_router_project(lib, want, change):
    assert project(lib, **change) == want


@pytest.mark.parametrize("want,change", SIZES + [(INVALID, {n: None}) for n in ("d", "x", "w", "ws")] +
                         [(INVALID, {n: at(8, 4)}) for n in ("d", "x", "w", "dres", "dx", "dw", "ws")] + [(SMALL, dict(size=15)),
                          (INVALID, dict(dw=None, w=None)), (INVALID, dict(dx=None, x=None)), (INVALID, dict(dw=None, d=None)), (INVALID, dict(dw=None, ws=None)),
                          (SMALL, dict(dw=None, size=15))])
def test_router_project_backward(lib, want, change):
    assert project_backward(lib, **change) == want


def test_router_project_of_nothing(lib):
    assert project(lib, T=0, x=None, w=None, logits=None, ws=None, size=0) == 0
    assert project_backward(lib, T=0, dw=None, d=None, x=None, ws=None) == 0
    assert project_backward(lib, dw=None, dx=None, x=None, w=None, ws=None) == 0
    assert moe.moe_router_project_workspace_bytes(0, 96, 24) >= 16
    with pytest.raises(moe.MoeError) as e:
        moe.moe_router_project_workspace_bytes(4, 96, 300)
    assert e.value.status == SHAPE
    assert lib.moe_router_project_workspace_bytes(4, 96, 24, None) == INVALID


# ---- orthogonal updates ----

def orth(lib, B=2, M=40, N=72, dtype=1, u=at(1), steps=5, coefs=None, eps=1e-7, out=at(2), ws=at(3), size=HUGE):
    kept = (ctypes.c_float * len(coefs))(*coefs) if coefs is not None else None
    return lib.moe_orthogonalize(B, M, N, dtype, u, steps, ctypes.addressof(kept) if coefs is not None else None, eps, out, ws, size, None)


def step(lib, B=2, M=40, N=72, dtype=1, g=at(1), m=at(2), w=at(3), master=None, mu=0.9, nesterov=1, lr=0.1, wd=0.0, scale=1.0, steps=5, eps=1e-7,
         m_out=at(5), w_out=at(6), ws=at(7), size=HUGE):
    return lib.moe_muon_step(B, M, N, dtype, g, m, w, master, mu, nesterov, lr, wd, scale, steps, None, eps, m_out, w_out, ws, size, None)


MATRICES = [(SHAPE, dict(B=-1)), (SHAPE, dict(M=0)), (SHAPE, dict(N=0)), (SHAPE, dict(M=(1 << 18) + 1)), (SHAPE, dict(M=32769, N=32769)),
            (SHAPE, dict(M=16384, N=131072)), (INVALID, dict(dtype=2)), (INVALID, dict(steps=0)), (INVALID, dict(steps=17)), (INVALID, dict(eps=0.0)),
            (INVALID, dict(eps=NAN)), (INVALID, dict(eps=INF)), (INVALID, dict(ws=None)), (INVALID, dict(ws=at(9, 8))), (SMALL, dict(size=1000))]


@pytest.mark.parametrize("want,change", MATRICES + [
    (INVALID, dict(u=None)), (INVALID, dict(out=None)), (INVALID, dict(u=at(1, 2))), (INVALID, dict(out=at(2, 8))), (INVALID, dict(out=at(1, 16))),
    (INVALID, dict(steps=1, coefs=(NAN, 0, 0))), (INVALID, dict(steps=1, coefs=(40, 0, 0))), (INVALID, dict(steps=1, coefs=(1, -3000, 3000))),
    (INVALID, dict(steps=4, coefs=(3, 0, 0) * 4))])
def test_orthogonalize(lib, want, change):
    assert orth(lib, **change) == want


@pytest.mark.parametrize("want,change", MATRICES + [
    *[(INVALID, {n: None}) for n in ("g", "m", "w", "m_out", "w_out")], *[(INVALID, {n: at(8, 4)}) for n in ("g", "m", "w", "m_out", "w_out", "master")],
    *[(INVALID, {n: NAN}) for n in ("mu", "lr", "wd", "scale")], (INVALID, dict(lr=INF)), (INVALID, dict(nesterov=2)),
    # arrays that share a part, or that a later matrix's inputs would be found overwritten in
    (INVALID, dict(m_out=at(2, 16))), (INVALID, dict(m_out=at(1))), (INVALID, dict(m_out=at(3))), (INVALID, dict(w_out=at(5))),
    (INVALID, dict(w_out=at(3, 32))), (INVALID, dict(w_out=at(1))), (INVALID, dict(w_out=at(2))), (INVALID, dict(master=at(6))),
    (INVALID, dict(master=at(5))), (INVALID, dict(master=at(1))), (INVALID, dict(master=at(2)))])
def test_muon_step(lib, want, change):
    assert step(lib, **change) == want


def test_no_matrices(lib):
    assert orth(lib, B=0, u=None, out=None, ws=None, size=0) == 0
    assert step(lib, B=0, g=None, m=None, w=None, m_out=None, w_out=None, ws=None, size=0) == 0
    assert lib.moe_muon_workspace_bytes(1, 4, 4, 1, None) == INVALID
    assert moe.moe_muon_workspace_bytes(0, 4, 4, torch.bfloat16) >= 0


def test_workspace_of_many_matrices_is_that_of_a_group():
    one = moe.moe_muon_workspace_bytes(1, 7168, 4096, torch.bfloat16)
    many = moe.moe_muon_workspace_bytes(1000, 7168, 4096, torch.bfloat16)
    assert one < many < 5 << 30
    assert moe.moe_muon_workspace_bytes(1000, 4096, 7168, torch.bfloat16) == many
    assert moe.moe_muon_workspace_bytes(4, 100, 90, torch.float32) > moe.moe_muon_workspace_bytes(4, 100, 90, torch.bfloat16)


# ---- the binding's own checks ----

def test_binding_checks_tensors():
    sc = moe.make_scores()
    with pytest.raises(ValueError, match="score"):
        moe.make_scores("tanh")
    shape = moe.make_shape(4, 64, 64, 8, 8, 0, 2, torch.bfloat16)
    saved = moe.alloc_saved(shape, device="cpu")
    with pytest.raises(ValueError, match="logits"):
        moe.moe_route_scores(shape, sc, torch.zeros(4, 8), None, saved, torch.zeros(1 << 20, dtype=torch.uint8))
    with pytest.raises(ValueError, match="logits"):
        moe.moe_route_scores_backward(sc, torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2), None, torch.zeros(4, 8))
    with pytest.raises(ValueError, match="bias"):
        moe.moe_bias_update(torch.zeros(8, dtype=torch.int32), 0.1, torch.zeros(8), torch.zeros(8))
    with pytest.raises(ValueError, match="x"):
        moe.moe_router_project(torch.zeros(4, 64), torch.zeros(64, 8), torch.zeros(4, 8), None)
    with pytest.raises(ValueError, match="x"):
        moe.moe_router_project(torch.zeros(4, 64, dtype=torch.float16), torch.zeros(64, 8), torch.zeros(4, 8), None)
    with pytest.raises(ValueError, match="w"):
        moe.moe_router_project(torch.zeros(4, 64), torch.zeros(64), torch.zeros(4, 8), None)
    with pytest.raises(ValueError, match="u"):
        moe.moe_orthogonalize(torch.zeros(1, 4, 4), torch.zeros(1, 4, 4), None)
    with pytest.raises(ValueError, match="g"):
        moe.moe_muon_step(torch.zeros(4, 4), None, None, None, None, None, lr=0.1)
    with pytest.raises(ValueError, match="coefs"):
        moe.binding._coefficients([(1.0, 2.0, 3.0)], 2)
    assert moe.binding._coefficients(None, 5) is None
