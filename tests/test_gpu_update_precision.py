"""What the orthogonal updates lose to rounding, held to what the documented roundings lose on the same matrices (update_emulation.py): operands of 11
bits in bf16 storage, of 22 in fp32, sums in fp32.  Whole matrices, and every 64 x 64 of them.

The kernel's roundings fall elsewhere than the emulation's (other scales, another order inside the sums), so the errors differ, but thousands of them
make up each norm: their sizes agree.  Allowed is four times the emulated error, beside the result's own rounding to its storage type: a factor
of two for the matrix cores' sums inside an instruction, which the emulation has exact, and two for a matrix whose roundings happen to fall badly."""
import pytest
import torch

import paper_2605_23764_amd as moe
import update_emulation as em
from block_common import HALF, TORCH

pytestmark = pytest.mark.gpu


def _blocks(e, side=64):
    """Norms of the 64 x 64 blocks."""
    M, N = e.shape
    p = torch.nn.functional.pad(e, (0, -N % side, 0, -M % side))
    return torch.linalg.vector_norm(p.view(p.shape[0] // side, side, p.shape[1] // side, side), dim=(1, 3))


def _hold(got, u, dtype, what, **how):
    want = em.orthogonalize(u, **how)
    lost = em.orthogonalize(u, **how, **em.STORED[dtype]) - want
    err, half = got.double() - want, HALF[dtype]
    norm = torch.linalg.vector_norm
    allowed = 4 * norm(lost) + half * (norm(want) + 4 * norm(lost))
    print(f"{what}: {norm(err) / norm(want):.2e} of the norm, emulated {norm(lost) / norm(want):.2e}, allowed {allowed / norm(want):.2e}", flush=True)
    assert norm(err) <= allowed
    b = _blocks(err) - half * _blocks(want)
    assert (b <= 4 * _blocks(lost).max() * (1 + half)).all(), (b.max(), _blocks(lost).max())
    return norm(err) / norm(want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,M,N", [(1, 200, 330), (1, 330, 200), (3, 64, 64), (2, 100, 1000), (2, 512, 512), (1, 257, 700), (1, 1000, 1570)])
def test_singular_values_down_to_a_hundredth(n, M, N, dtype):
    """The figures that the header gives for such matrices: up to 5e-3 and 5e-6 of the result's norm.  (Operands of 11 bits alone leave 1.9e-3 to
    4.0e-3 here, the result's own rounding to bf16 1.7e-3.)"""
    u = torch.stack([em.spectrum(M, N, 0.01, 7 * M + e) for e in range(n)]).cuda().to(TORCH[dtype])
    out = torch.full_like(u, float("nan"))
    moe.moe_orthogonalize(u, out, moe.alloc_muon_workspace(n, M, N, TORCH[dtype]))
    for e in range(n):
        share = _hold(out[e], u[e], dtype, f"{M} x {N} {dtype}")
        assert share <= {"bf16": 5e-3, "f32": 5e-6}[dtype]


# Sizes whose products take whole tiles of 256, quarters of what is left over, shares along the reduction, tiles of 128 and of 64
@pytest.mark.parametrize("dtype,n,M,N", [("bf16", 26, 1000, 1570), ("bf16", 26, 1570, 1000), ("f32", 7, 1000, 1570), ("f32", 7, 1570, 1000), ("bf16", 270, 130, 200),
                                         ("f32", 270, 130, 200), ("f32", 100, 300, 500), ("bf16", 5, 700, 1100), ("f32", 5, 700, 1100), ("bf16", 1, 256, 4096),
                                         ("f32", 1, 256, 4096), ("bf16", 9, 640, 640)])
def test_every_way_through_the_tiles(dtype, n, M, N):
    """Strong directions over a broad rest, as momentum has them; the first, a middle and the last matrix, whose tiles are left over from whole rounds."""
    g = torch.Generator("cuda").manual_seed(M + n)
    k = max(1, min(M, N) // 16)
    u = torch.empty(n, M, N, dtype=TORCH[dtype], device="cuda")
    for e in range(n):
        u[e] = torch.randn(M, k, generator=g, device="cuda") @ torch.randn(k, N, generator=g, device="cuda") * k ** -0.5 + torch.randn(M, N, generator=g, device="cuda")
    out = torch.full_like(u, float("nan"))
    moe.moe_orthogonalize(u, out, moe.alloc_muon_workspace(n, M, N, TORCH[dtype]))
    for e in sorted({0, n // 2, n - 1}):
        _hold(out[e], u[e], dtype, f"{n} x {M} x {N} {dtype}, {e}")


@pytest.mark.parametrize("dtype,wrong", [("bf16", dict(operand_bits=8)), ("f32", dict(em.STORED["f32"], pairs_of=((0, 0),))),
                                         ("f32", dict(em.STORED["f32"], pairs_of=((0, 0), (1, 0))))])
def test_the_measure_sees_coarser_operands(dtype, wrong):
    """Planted in the emulation: operands of 8 bits, products without a rest."""
    u = em.spectrum(200, 330, 0.01, 3).cuda()
    with pytest.raises(AssertionError):
        _hold(em.orthogonalize(u, **wrong).to(TORCH[dtype]), u, dtype, "planted")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,N", [(48, 100), (100, 48), (1, 90), (90, 1), (300, 200), (200, 300)])
def test_one_value_that_is_none_spoils_its_matrix_and_no_other(M, N, dtype):
    """A NaN or an infinity anywhere: every value of the result is NaN, on either side of M = N."""
    u = torch.randn(6, M, N, generator=torch.Generator("cuda").manual_seed(M), device="cuda").to(TORCH[dtype])
    ws = moe.alloc_muon_workspace(6, M, N, TORCH[dtype])
    want = torch.empty_like(u)
    moe.moe_orthogonalize(u, want, ws)
    u[1, M // 2, N // 3], u[3, M - 1, N - 1], u[4, 0, 0] = float("nan"), float("inf"), -float("inf")
    for steps in (1, 5):
        out = torch.full_like(u, 7.0)
        moe.moe_orthogonalize(u, out, ws, steps=steps)
        assert torch.isnan(out[[1, 3, 4]]).all(), steps
        assert torch.isfinite(out[[0, 2, 5]]).all()
    assert torch.equal(out[[0, 2, 5]], want[[0, 2, 5]])
