"""The router's projection and its backward on the GPU, against fp64: odd sizes, one row to many, fewer columns than a tile, several splits
along the reduction, outputs over inputs, missing outputs."""
import numpy as np
import pytest
import torch

import paper_2605_23764_amd as moe
from block_common import HALF, TORCH, U, close, f64

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1, 1), (1, 7168, 256), (2, 33, 5), (3, 40, 8), (17, 129, 24), (31, 1001, 60), (64, 64, 64), (100, 320, 128), (129, 127, 129), (200, 2048, 16),
          (333, 65, 255), (1500, 1001, 24), (130, 5000, 3), (5000, 96, 160)]


def _inputs(T, H, E, dtype, seed):
    r = np.random.default_rng(seed)
    x = torch.from_numpy(r.normal(size=(T, H)).astype(np.float32)).cuda().to(TORCH[dtype])
    w = torch.from_numpy((r.normal(size=(H, E)) * np.exp(r.normal(size=(H, E)))).astype(np.float32)).cuda()
    d = torch.from_numpy((r.normal(size=(T, E)) * 10.0 ** r.uniform(-6, 0, size=(T, 1))).astype(np.float32)).cuda()
    dres = torch.from_numpy(r.normal(size=(T, H)).astype(np.float32)).cuda().to(TORCH[dtype])
    return x, w, d, dres


def _bound(K, magnitude, products, left_out):
    """A sum of K terms by MFMAs of 16 (each adds its own sums to one element: at most 16 roundings inside, one outside), `products`
    of them per term, up to 256 partial sums joined by four waves; twice over for the order inside."""
    return (2 * (products * (K / 16 + 1) + 16 + 64 + 4) * U + left_out) * magnitude


def _new(*shape, dtype=torch.float32):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,E", SHAPES)
def test_forward_and_backward(T, H, E, dtype):
    print(f"project T={T} H={H} E={E} {dtype}", flush=True)
    x, w, d, dres = _inputs(T, H, E, dtype, T + H + E)
    X, W, D, R = (f64(t) for t in (x, w, d, dres))
    both = dtype == "f32"
    ws = torch.full((moe.moe_router_project_workspace_bytes(T, H, E),), 255, dtype=torch.uint8, device="cuda")
    logits = _new(T, E)
    moe.moe_router_project(x, w, logits, ws)
    close(logits, X @ W, _bound(H, np.abs(X) @ np.abs(W), 6 if both else 3, 2.0 ** -21 if both else 0.0) + U * np.abs(X @ W), "logits")
    dx, dw = _new(T, H, dtype=TORCH[dtype]), _new(H, E)
    ws.fill_(255)
    moe.moe_router_project_backward(d, x, w, dres, dx, dw, ws)
    close(dw, X.T @ D, _bound(T, np.abs(X).T @ np.abs(D), 6 if both else 3, 2.0 ** -21 if both else 0.0) + U * np.abs(X.T @ D), "dw")
    raw, size = D @ W.T, np.abs(D) @ np.abs(W).T
    e = _bound(E, size, 6 if both else 3, 2.0 ** -21 if both else 2.0 ** -13)
    close(dx, R + raw, e + (U + HALF[dtype]) * (np.abs(R + raw) + e), "dx")
    # without the other gradient, the residual's part, and over the inputs
    alone, dw2 = _new(T, H, dtype=TORCH[dtype]), _new(H, E)
    moe.moe_router_project_backward(d, x, w, dres, alone, None, ws)
    moe.moe_router_project_backward(d, x, w, None, None, dw2, ws)
    assert torch.equal(alone, dx) and torch.equal(dw2, dw)
    moe.moe_router_project_backward(d, x, w, None, alone, None, ws)
    close(alone, raw, e + (U + HALF[dtype]) * (np.abs(raw) + e), "dx without a residual")
    over = dres.clone()
    moe.moe_router_project_backward(d, x, w, over, over, None, ws)
    assert torch.equal(over, dx)
    over = x.clone()
    moe.moe_router_project_backward(d, over, w, dres, over, dw2, ws)
    assert torch.equal(over, dx) and torch.equal(dw2, dw)


def test_no_tokens():
    x, w, d, _ = _inputs(1, 40, 8, "bf16", 0)
    dw = _new(40, 8)
    ws = moe.alloc_router_project_workspace(0, 40, 8)
    moe.moe_router_project(x[:0], w, torch.empty(0, 8, device="cuda"), ws)
    moe.moe_router_project_backward(d[:0], x[:0], w, None, x[:0], dw, ws)
    assert (dw == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_small_and_large_values(dtype):
    """Values over the whole range of exponents that a product can have: the pieces are exact."""
    T, H, E = 40, 96, 24
    r = np.random.default_rng(4)
    x = torch.from_numpy((r.normal(size=(T, H)) * 2.0 ** r.integers(-30, 30, size=(T, 1))).astype(np.float32)).cuda().to(TORCH[dtype])
    w = torch.from_numpy((r.normal(size=(H, E)) * 2.0 ** r.integers(-30, 30, size=(1, E))).astype(np.float32)).cuda()
    logits = _new(T, E)
    moe.moe_router_project(x, w, logits, moe.alloc_router_project_workspace(T, H, E))
    X, W = f64(x), f64(w)
    close(logits, X @ W, _bound(H, np.abs(X) @ np.abs(W), 6, 2.0 ** -21) + U * np.abs(X @ W), "logits")


def test_a_row_spoils_no_other():
    x, w, d, _ = _inputs(200, 96, 24, "bf16", 9)
    logits, want = _new(200, 24), _new(200, 24)
    ws = moe.alloc_router_project_workspace(200, 96, 24)
    moe.moe_router_project(x, w, want, ws)
    x[77] = float("nan")
    x[150, 3] = float("inf")
    moe.moe_router_project(x, w, logits, ws)
    keep = torch.ones(200, dtype=torch.bool, device="cuda")
    keep[[77, 150]] = False
    assert torch.equal(logits[keep], want[keep]) and torch.isnan(logits[77]).all() and not torch.isfinite(logits[150]).any()


def test_gradient_against_differences():
    T, H, E = 6, 20, 9
    x, w, d, _ = _inputs(T, H, E, "f32", 2)
    dx, dw, ws = _new(T, H), _new(H, E), moe.alloc_router_project_workspace(T, H, E)
    moe.moe_router_project_backward(d, x, w, None, dx, dw, ws)

    def loss(a, b):
        out = _new(T, E)
        moe.moe_router_project(a, b, out, ws)
        return (f64(out) * f64(d)).sum()

    # a linear map: a whole step is as good as a small one; the difference of two fp32 results
    size = (np.abs(f64(x)) @ np.abs(f64(w)) * np.abs(f64(d))).sum() + (np.abs(f64(d))).sum() * np.abs(f64(w)).max()
    for grad, which in ((dx, 0), (dw, 1)):
        for at in ((0, 0), (3, 7), (5, 8)):
            a, b = x.clone(), w.clone()
            (a, b)[which][at] += 1.0
            step = f64((a, b)[which][at] - (x, w)[which][at])
            assert abs((loss(a, b) - loss(x, w)) / step - f64(grad)[at]) <= 100 * U * size / abs(step) + 2.0 ** -20 * abs(f64(grad)[at])


def test_same_bits_again_and_from_a_graph():
    T, H, E = 700, 300, 60
    x, w, d, dres = _inputs(T, H, E, "bf16", 1)
    out = [_new(T, E), _new(T, H, dtype=torch.bfloat16), _new(H, E)]
    ws = moe.alloc_router_project_workspace(T, H, E)

    def step():
        moe.moe_router_project(x, w, out[0], ws)
        moe.moe_router_project_backward(d, x, w, dres, out[1], out[2], ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for i in range(4):
        for t, v in zip((x, w, d, dres), _inputs(T, H, E, "bf16", 30 + i % 3)):
            t.copy_(v)
        for t in out:
            t.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, out))
