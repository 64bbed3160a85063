"""Orthogonal updates on the GPU, against the fp64 oracle: either side longer, one row to several tiles, odd sizes, many matrices, both storage
types, momentum and weights in place and apart."""
import numpy as np
import pytest
import torch

import paper_2605_23764_amd as moe
from block_common import HALF, TORCH, U, close, f64
from oracle import router_oracle as ro

pytestmark = pytest.mark.gpu

BITS = {"bf16": 2.0 ** -11, "f32": 2.0 ** -22 + 2.0 ** -22}   # an operand's rounding: fp16; a pair of fp16, and the product of their rests
LIP = 3.9                                                    # largest slope of the usual polynomial up to 1.2, the first step's 3.45 among them
SHAPES = [(1, 1, 1), (2, 1, 7), (2, 9, 1), (1, 64, 64), (3, 65, 130), (2, 200, 330), (1, 330, 200), (2, 300, 300), (1, 257, 700), (1, 700, 257), (1, 5, 1000),
          (2, 576, 320)]


def _bound(u, dtype, steps=5, coefs=None, eps=1e-7, lip=LIP):
    """How far the result may be off, in the Frobenius norm.  With d an operand's relative rounding, a step adds
      of A:  (|b| + 2 |c| |A|2) (d max diag A |X|F + d |A off|F |X|2)      (a diagonal matrix times X, and any other)
      of B:  d max diag B |X|F + d |B off|F |X|2
      of the next X: d |X'|F
    the same with K / 8 + 8 roundings of an fp32 sum in front of each, and takes what it was given on by the polynomial's largest slope
    (the largest divided difference of an odd function on the singular values)."""
    x = f64(u) if isinstance(u, torch.Tensor) else u
    x = x if x.shape[0] <= x.shape[1] else x.T
    x = x / (np.sqrt((x * x).sum()) + eps)
    d0 = BITS[dtype]
    err = (d0 + 4 * U) * np.sqrt((x * x).sum())
    for i in range(steps):
        a, b, c = ro.USUAL if coefs is None else coefs[i]
        A = x @ x.T
        B = a * np.eye(len(A)) + b * A + c * A @ A
        d = d0 + (max(x.shape) / 8 + 8) * U
        two, fro = np.linalg.norm(x, 2), np.linalg.norm(x)
        off = lambda m: np.linalg.norm(m - np.diag(np.diag(m)))  # noqa: E731
        part = lambda m: d * (np.abs(np.diag(m)).max() * fro + off(m) * two)  # noqa: E731
        noise = (abs(b) + 2 * abs(c) * two ** 2) * part(A) + part(np.abs(B) + abs(b) * np.abs(A) + abs(c) * np.abs(A) @ np.abs(A))
        x = B @ x
        err = lip * err + noise + d * np.linalg.norm(x)
    return x, err


def _u(n, M, N, seed, size=1e-3):
    r = np.random.default_rng(seed)
    k = max(1, min(M, N) // 8)
    return (r.normal(size=(n, M, k)) @ r.normal(size=(n, k, N)) / np.sqrt(k) + r.normal(size=(n, M, N))) * size


def _dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(TORCH[dtype])


def _ws(n, M, N, dtype):
    return torch.full((moe.moe_muon_workspace_bytes(n, M, N, TORCH[dtype]),), 255, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,M,N", SHAPES)
def test_orthogonalize(n, M, N, dtype):
    print(f"orthogonalize {n} x {M} x {N} {dtype}", flush=True)
    u = _dev(_u(n, M, N, M + N), dtype)
    out = torch.full_like(u, float("nan"))
    ws = _ws(n, M, N, dtype)
    moe.moe_orthogonalize(u, out, ws)
    got = f64(out)
    for e in range(n):
        want = ro.orthogonalize(f64(u)[e])
        _, err = _bound(u[e], dtype)
        off = np.linalg.norm(got[e] - want)
        allowed = err + HALF[dtype] * (np.linalg.norm(want) + err)
        assert off <= allowed, f"matrix {e}: {off:.3g} > {allowed:.3g}"
        # what the worst case leaves out: roundings are independent, so their sum stays far below it
        assert off <= 0.5 * err + HALF[dtype] * np.linalg.norm(want) or min(M, N) < 16
    again = u.clone()
    moe.moe_orthogonalize(again, again, ws)
    assert torch.equal(again, out)


@pytest.mark.parametrize("M,N", [(1000, 1570), (1570, 1000)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_whole_rounds_and_what_is_left_over(M, N, dtype):
    """Products of several rounds of the chip: whole tiles, quarters of the last, shares along the reduction; the first, a middle and the last
    matrix against the oracle, all against each other's spectra."""
    n = 26 if dtype == "bf16" else 7
    print(f"orthogonalize {n} x {M} x {N} {dtype}", flush=True)
    g = torch.Generator("cuda").manual_seed(M)
    u = (torch.randn(n, M, 40, generator=g, device="cuda") @ torch.randn(n, 40, N, generator=g, device="cuda") * 40 ** -0.5
         + torch.randn(n, M, N, generator=g, device="cuda")).to(TORCH[dtype])
    out = torch.full_like(u, float("nan"))
    moe.moe_orthogonalize(u, out, _ws(n, M, N, dtype))
    assert torch.isfinite(out).all()
    for e in (0, n // 2, n - 1):
        want, err = _bound(u[e], dtype)
        want = want if M <= N else want.T
        off = np.linalg.norm(f64(out)[e] - want)
        assert off <= 0.5 * err + HALF[dtype] * (np.linalg.norm(want) + err), f"matrix {e}: {off:.3g}, {err:.3g}"
    one = torch.empty_like(u[:1])
    ws = _ws(1, M, N, dtype)
    for e in range(n):                                                # alone a matrix takes other tiles: the same up to roundings
        moe.moe_orthogonalize(u[e:e + 1], one, ws)
        assert torch.linalg.vector_norm((one[0] - out[e]).float()) <= (err + HALF[dtype] * np.linalg.norm(want)), e


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_coefficients_and_steps(dtype):
    u = _dev(_u(2, 70, 150, 3), dtype)
    out, ws = torch.empty_like(u), _ws(2, 70, 150, dtype)
    coefs = [(8.0, -22.0, 16.0), (4.0, -2.9, 0.55), (1.9, -1.3, 0.4)]
    slopes = []
    top = 1.0
    for a, b, c in coefs:
        s = np.linspace(0, top, 2001)
        slopes.append(max(np.abs(a + 3 * b * s ** 2 + 5 * c * s ** 4).max(), np.abs(a + b * s ** 2 + c * s ** 4).max()))
        top = np.abs(a * s + b * s ** 3 + c * s ** 5).max()
    for n in (1, 3):
        moe.moe_orthogonalize(u, out, ws, steps=n, coefs=coefs[:n])
        for e in range(2):
            want = ro.orthogonalize(f64(u)[e], n, coefs)
            _, err = _bound(u[e], dtype, n, coefs, lip=max(slopes[:n]))
            assert np.linalg.norm(f64(out)[e] - want) <= err + HALF[dtype] * (np.linalg.norm(want) + err)
    # the eps of a matrix that is not much larger
    moe.moe_orthogonalize(u, out, ws, steps=2, eps=0.5)
    want = ro.orthogonalize(f64(u)[0], 2, eps=0.5)
    _, err = _bound(u[0], dtype, 2, eps=0.5)
    assert np.linalg.norm(f64(out)[0] - want) <= err + HALF[dtype] * (np.linalg.norm(want) + err)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_extreme_matrices(dtype):
    """Zeros, one value, one direction, values at both ends of the range, NaN and infinities: each by itself."""
    M, N = 48, 100
    r = np.random.default_rng(0)
    base = r.normal(size=(M, N))
    us = [np.zeros((M, N)), np.where((np.arange(M)[:, None] == 3) & (np.arange(N) == 5), -2e-5, 0.0), np.outer(r.normal(size=M), r.normal(size=N)),
          base * 1e30, base * 1e-30, base, base, base]
    u = _dev(np.stack(us), dtype)
    u[5, 7, 9], u[6, 0, 0] = float("nan"), float("inf")
    out, ws = torch.empty_like(u), _ws(len(us), M, N, dtype)
    moe.moe_orthogonalize(u, out, ws, eps=1e-37)
    assert (out[0] == 0).all() and torch.isnan(out[5]).all() and torch.isnan(out[6]).any()
    for e in (1, 2, 3, 4, 7):
        want = ro.orthogonalize(f64(u)[e], eps=float(np.float32(1e-37)))
        _, err = _bound(u[e], dtype, eps=1e-37)
        assert np.linalg.norm(f64(out)[e] - want) <= err + HALF[dtype] * (np.linalg.norm(want) + err), e
    moe.moe_orthogonalize(u, out, ws, eps=1.0)                        # a matrix of 1e-30 beside an eps of 1: nothing left of it
    assert np.abs(f64(out)[4]).max() < 1e-26


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,M,N", [(1, 3, 5), (3, 130, 70), (2, 96, 320)])
def test_step(n, M, N, dtype):
    g, m, w = _dev(_u(n, M, N, 1), dtype), _dev(_u(n, M, N, 2), "f32"), _dev(_u(n, M, N, 3, 1.0), dtype)
    ws = _ws(n, M, N, dtype)
    lr, mu, wd, scale = 0.05, 0.9, 0.2, 1.5
    for nesterov in (True, False):
        m_out, w_out = torch.full_like(m, float("nan")), torch.full_like(w, float("nan"))
        moe.moe_muon_step(g, m, w, m_out, w_out, ws, lr=lr, mu=mu, nesterov=nesterov, weight_decay=wd, scale=scale)
        f = lambda v: float(np.float32(v))  # noqa: E731
        master = f64(w).astype(np.float32)
        dev_master, w_copy = torch.from_numpy(master).cuda(), torch.full_like(w, float("nan"))
        m_same = m.clone()
        moe.moe_muon_step(g, m_same, None, m_same, w_copy, ws, lr=lr, mu=mu, nesterov=nesterov, weight_decay=wd, scale=scale, master=dev_master)
        assert torch.equal(m_same, m_out)
        same = w.clone()
        moe.moe_muon_step(g, m, same, m_out, same, ws, lr=lr, mu=mu, nesterov=nesterov, weight_decay=wd, scale=scale)
        assert torch.equal(same, w_out) and torch.equal(w_copy, w_out) and torch.equal(dev_master.to(w.dtype), w_out)
        for e in range(n):
            M1, W1 = ro.muon_step(f64(g)[e], f64(m)[e], f64(w)[e], f(lr), f(mu), nesterov, f(wd), f(scale))
            close(m_out[e], M1, 2 * U * (np.abs(f(mu) * f64(m)[e]) + np.abs(M1)), "momentum")
            u = f64(g)[e] + f(mu) * M1 if nesterov else M1
            _, err = _bound(u, dtype)
            err += LIP ** 5 * 6 * U                                     # of u itself: a few roundings, of norm 1 after the division
            off = np.linalg.norm(f64(dev_master)[e] - W1)
            assert off <= f(lr) * f(scale) * err + 4 * U * np.linalg.norm(W1), (e, off)
            off = np.linalg.norm(f64(w_out)[e] - W1)
            assert off <= f(lr) * f(scale) * err + (HALF[dtype] + 4 * U) * np.linalg.norm(W1), (e, off)


@pytest.mark.parametrize("M,N", [(130, 200), (200, 130), (260, 203)])
@pytest.mark.parametrize("master", [False, True], ids=["weights", "master"])
def test_step_of_many_is_each_ones(M, N, master):
    """As many matrices as make whole tiles: weights and fp32 ones, fetched ahead, apart and in place, sides that end inside a block and rows
    at odd addresses; the bits of each alone, and nothing beside them."""
    n = 270
    gen = torch.Generator("cuda").manual_seed(M)
    g, w = (torch.randn(n, M, N, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    m, top = torch.randn(n, M, N, generator=gen, device="cuda"), torch.randn(n, M, N, generator=gen, device="cuda")
    ws, ws1 = _ws(n, M, N, "bf16"), _ws(1, M, N, "bf16")
    kw = dict(lr=0.3, mu=0.9, weight_decay=0.1)
    rim = torch.full((n * M * N + 512,), 7.0, dtype=torch.bfloat16, device="cuda")
    out = rim[256:-256].view(n, M, N)
    m_out, big = torch.empty_like(m), top.clone()
    moe.moe_muon_step(g, m, None if master else w, m_out, out, ws, master=big if master else None, **kw)
    assert (rim[:256] == 7).all() and (rim[-256:] == 7).all()
    same = w.clone()
    if not master:
        moe.moe_muon_step(g, m, same, m_out, same, ws, **kw)
        assert torch.equal(same, out)
    for e in (0, 1, 100, 255, 256, n - 1):
        one, t, m1 = torch.empty(1, M, N, dtype=torch.bfloat16, device="cuda"), top[e:e + 1].clone(), torch.empty(1, M, N, device="cuda")
        moe.moe_muon_step(g[e:e + 1].clone(), m[e:e + 1].clone(), None if master else w[e:e + 1].clone(), m1, one, ws1, master=t if master else None, **kw)
        assert torch.equal(one[0], out[e]) and torch.equal(m1[0], m_out[e]), e
        if master:
            assert torch.equal(t[0], big[e]) and torch.equal(big[e].to(torch.bfloat16), out[e]), e


@pytest.mark.parametrize("n,M,N", [(270, 130, 200), (270, 260, 203), (270, 70, 300), (270, 3, 90), (100, 300, 500)])
def test_fp32_of_many_is_each_ones(n, M, N):
    """fp32 matrices as many as make whole tiles, whose reductions are two to sixteen steps long, and what is left over of them in quarters: the
    oracle's, and in whole tiles the bits of each alone; weights in place, and fp32 ones beside a copy."""
    u = _dev(_u(n, M, N, M + n), "f32")
    out, ws, ws1 = torch.full_like(u, float("nan")), _ws(n, M, N, "f32"), _ws(1, M, N, "f32")
    moe.moe_orthogonalize(u, out, ws)
    w = torch.randn(n, M, N, generator=torch.Generator("cuda").manual_seed(M), device="cuda")
    m, m_out, same, top, copy = torch.ones_like(u), torch.empty_like(u), w.clone(), w.clone(), torch.full_like(u, float("nan"))
    kw = dict(lr=0.3, mu=0.9, weight_decay=0.1)
    moe.moe_muon_step(u, m, same, m_out, same, ws, **kw)
    moe.moe_muon_step(u, m, None, m_out, copy, ws, master=top, **kw)
    assert torch.equal(same, top) and torch.equal(same, copy)
    one, m1 = torch.empty(1, M, N, device="cuda"), torch.empty(1, M, N, device="cuda")
    # The last 14 of 270 are what is left over of a round of 256, and sums of eight steps are dealt out in two shares: added up in another
    # order, so within the bound of each (its term of K / 8 + 8 roundings), not the same bits.
    for e in (0, 1, n // 2, n - 2, n - 1):
        moe.moe_orthogonalize(u[e:e + 1].clone(), one, ws1)
        _, err = _bound(u[e], "f32")
        assert torch.equal(one[0], out[e]) or (e >= 256 and torch.linalg.vector_norm(one[0] - out[e]) <= 2 * err), e
        moe.moe_muon_step(u[e:e + 1].clone(), m[:1].clone(), w[e:e + 1].clone(), m1, one, ws1, **kw)
        assert torch.equal(m1[0], m_out[e]), e
        _, err = _bound(f64(u)[e] + f64(torch.tensor(0.9)) * f64(m_out)[e], "f32")
        assert torch.equal(one[0], same[e]) or (e >= 256 and torch.linalg.vector_norm(one[0] - same[e]) <= 0.3 * 2 * err + 4 * U * float(torch.linalg.vector_norm(same[e]))), e
    for e in (0, n - 1):
        want, err = _bound(u[e], "f32")
        want = want if M <= N else want.T
        off = np.linalg.norm(f64(out)[e] - want)
        assert off <= err + HALF["f32"] * (np.linalg.norm(want) + err), (e, off, err)


def test_more_matrices_than_a_group():
    """Beyond the matrices that are worked on at a time, each is what it is alone."""
    n, M, N = 16500, 6, 20
    u = torch.randn(n, M, N, generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    out, ws = torch.full_like(u, float("nan")), _ws(n, M, N, "bf16")
    moe.moe_orthogonalize(u, out, ws)
    for e in (0, 1, 8249, 8250, 16384, 16499):
        one = torch.empty_like(u[:1])
        moe.moe_orthogonalize(u[e:e + 1], one, ws)
        assert torch.equal(one[0], out[e]), e
    assert not torch.isnan(out).any()


def test_transposed_matrix_has_the_transposed_update():
    u = _dev(_u(1, 150, 90, 5), "f32")
    a, b = torch.empty_like(u), torch.empty(1, 90, 150, device="cuda")
    ws = _ws(1, 150, 90, "f32")
    moe.moe_orthogonalize(u, a, ws)
    moe.moe_orthogonalize(u.transpose(1, 2).contiguous(), b, ws)
    assert (a.transpose(1, 2) - b).abs().max() < 1e-5


def test_same_bits_again_and_from_a_graph():
    n, M, N = 3, 200, 140
    g, m, w = (_dev(_u(n, M, N, i), t) for i, t in ((1, "bf16"), (2, "f32"), (3, "bf16")))
    ws = _ws(n, M, N, "bf16")

    def step():
        moe.moe_muon_step(g, m, w, m, w, ws, lr=0.02)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for i in range(4):
        g.copy_(_dev(_u(n, M, N, 10 + i), "bf16"))
        before = m.clone(), w.clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = m.clone(), w.clone()
        m.copy_(before[0]), w.copy_(before[1])
        step()
        torch.cuda.synchronize()
        assert torch.equal(m, got[0]) and torch.equal(w, got[1])


def test_streams_and_devices_memory():
    """On a stream of its own, whose inputs become right there only."""
    n, M, N = 2, 130, 200
    good, u = _dev(_u(n, M, N, 1), "bf16"), _dev(_u(n, M, N, 2), "bf16")
    want, out, ws = torch.empty_like(u), torch.empty_like(u), _ws(n, M, N, "bf16")
    moe.moe_orthogonalize(good, want, ws)
    busy = torch.randn(4096, 4096, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(8):
            busy = (busy @ busy) * 1e-2
        u.copy_(good)
    moe.moe_orthogonalize(u, out, ws, stream=s)
    s.synchronize()
    assert torch.equal(out, want)
