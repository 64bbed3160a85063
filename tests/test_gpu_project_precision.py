"""What the router's projection loses to rounding, block by block of its results, in the Frobenius norm.

Derivation.  With t the K terms of an element, a sum in fp32 is rounded once per matrix instruction (16 terms, `products` of them per term) and some 80
times where partial sums are joined, each by at most U of the partial sum, whose size is that of the root of the sum of t^2 where signs are
random: independent, they add up to U (n / 3)^0.5 |t|.  What the pieces leave out: 2^-24 of a product on average in fp32 (2^-21 at most), in dx in bf16
at most 2^-13, half of it on average and of one sign.  Allowed is twice that, and 3^0.5 for the instruction's own sums, four times it in blocks
of fewer than 64 elements, which average little; and the result's own rounding."""
import pytest
import torch

import paper_2605_23764_amd as moe
from block_common import HALF, TORCH, U

pytestmark = pytest.mark.gpu

SHAPES = [(1, 7168, 256), (3, 40, 8), (31, 1001, 60), (64, 64, 64), (129, 127, 129), (200, 2048, 16), (333, 65, 255), (1500, 1001, 24), (130, 5000, 3),
          (5000, 96, 160), (4096, 2048, 64), (4096, 4096, 256)]


def _inputs(T, H, E, dtype):
    g = torch.Generator("cuda").manual_seed(T + H + E)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")
    return normal(T, H).to(TORCH[dtype]), normal(H, E) * torch.exp(normal(H, E)), normal(T, E), normal(T, H).to(TORCH[dtype])


def _block_norms(e, rows=128, cols=64):
    p = torch.nn.functional.pad(e, (0, -e.shape[1] % cols, 0, -e.shape[0] % rows))
    return torch.linalg.vector_norm(p.view(p.shape[0] // rows, rows, p.shape[1] // cols, cols), dim=(1, 3))


def _hold(got, P, Q, products, left, add, half, what):
    """got against P Q (+ add) in 64 bits."""
    P, Q = P.double().contiguous(), Q.double().contiguous()
    sums = P @ Q
    want = sums if add is None else sums + add.double()
    err = _block_norms(got.double() - want)
    size = _block_norms((P * P @ (Q * Q)).sqrt())
    n = products * -(-P.shape[1] // 16) + 80
    elements = _block_norms(torch.ones_like(want)) ** 2
    factor = torch.where(elements < 64, 4.0, 2.0)
    allowed = factor * (U * n ** 0.5 * size + left / 2 * (size + _block_norms(sums))) + (half + 2 * U) * _block_norms(want)
    worst = torch.where(err == 0, 0.0, err / allowed).max().item()             # nothing but zeros: nothing is allowed
    print(f"{what}: {err.norm():.2e} against {_block_norms(want).norm():.2e}, worst block {worst:.2f} of what is allowed", flush=True)
    return worst


def _cases(T, H, E, dtype):
    x, w, d, dres = _inputs(T, H, E, dtype)
    f32 = dtype == "f32"
    products = 6 if f32 else 3
    return x, w, d, dres, dict(logits=(x, w, products, 2.0 ** -24 if f32 else 0.0, None, 0.0),
                               dw=(x.t(), d, products, 2.0 ** -24 if f32 else 0.0, None, 0.0),
                               dx=(d, w.t(), products, 2.0 ** -24 if f32 else 2.0 ** -13, dres, HALF[dtype]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,E", SHAPES)
def test_forward_and_backward(T, H, E, dtype):
    x, w, d, dres, cases = _cases(T, H, E, dtype)
    ws = moe.alloc_router_project_workspace(T, H, E)
    got = dict(logits=torch.empty(T, E, device="cuda"), dx=torch.empty_like(x), dw=torch.empty_like(w))
    moe.moe_router_project(x, w, got["logits"], ws)
    moe.moe_router_project_backward(d, x, w, dres, got["dx"], got["dw"], ws)
    for name, (P, Q, products, left, add, half) in cases.items():
        assert _hold(got[name], P, Q, products, left, add, half, f"{name} T={T} H={H} E={E} {dtype}") <= 1, name


def _high(v, n):
    """v cut off to n pieces of 8 bits."""
    out, rest = torch.zeros_like(v), v.clone()
    for _ in range(n):
        piece = (rest.view(torch.int32) & -65536).view(torch.float32)
        out, rest = out + piece, rest - piece
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,E", SHAPES)
def test_the_measure_sees_a_missing_piece(T, H, E, dtype):
    """Planted in the plain products: W of two pieces where it has three (logits), dlogits of two (dW)."""
    x, w, d, dres, cases = _cases(T, H, E, dtype)
    for name, wrong in (("logits", (x.double() @ _high(w, 2).double()).float()), ("dw", (x.double().t().contiguous() @ _high(d, 2).double()).float())):
        P, Q, products, left, add, half = cases[name]
        assert _hold(wrong, P, Q, products, left, add, half, f"planted, {name}") > 1, name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("power", [-100, -110, -115, -120, -125, -130, -140])
def test_values_near_the_least(power, dtype):
    """Of fp32 values below 2^-109 the multiples of 2^-133 in them count, here of W and dlogits (times large ones, so that sums are ordinary)."""
    T, H, E = 40, 96, 24
    x, w, d, _ = _inputs(T, H, E, dtype)
    x = (x.float() * 2.0 ** 60).to(TORCH[dtype])
    large = w * 2.0 ** 60
    w, d = ((t.double() * 2.0 ** power).float() for t in (w, d))
    cut = lambda v: torch.where(v.abs() < 2.0 ** -109, torch.trunc(v.double() * 2.0 ** 133) * 2.0 ** -133, v.double())  # noqa: E731
    logits, dx, dw = torch.empty(T, E, device="cuda"), torch.empty_like(x), torch.empty(H, E, device="cuda")
    ws = moe.alloc_router_project_workspace(T, H, E)
    moe.moe_router_project(x, w, logits, ws)
    moe.moe_router_project_backward(d, x, large, None, None, dw, ws)
    moe.moe_router_project_backward(d, x, large, None, dx, None, ws)
    f32 = dtype == "f32"
    for got, P, Q, left, half in ((logits, x, cut(w), 2.0 ** -24 * f32, 0.0), (dw, x.t(), cut(d), 2.0 ** -24 * f32, 0.0),
                                  (dx, cut(d), large.t(), 2.0 ** -24 if f32 else 2.0 ** -13, HALF[dtype])):
        assert _hold(got, P, Q, 6 if f32 else 3, left, None, half, f"2^{power} {dtype}") <= 1
