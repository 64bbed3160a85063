"""The block's update of its experts: gate and up by themselves or as one matrix, the factor from what a matrix takes in and gives out."""
import numpy as np
import pytest
import torch

import paper_2605_23764_amd as moe
from block_common import HALF, U, close, f64
from oracle import router_oracle as ro
from paper_2605_23764_amd.moe_block import MoeBlock
from test_gpu_muon import _bound

pytestmark = pytest.mark.gpu

LR, MU, WD = (float(np.float32(v)) for v in (0.05, 0.9, 0.1))


def _block(H, I, dtype, E=3, T=40):
    b = MoeBlock(T, H, I, E, 2, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, seed=3, scores=moe.make_scores("sigmoid"))
    b.counts.zero_()
    return b


def _gradients(b, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    for t in (b.dw_gate_up, b.dw_down):
        t.copy_(torch.randn(t.shape, generator=g, device="cuda") * 1e-3)


def _check(got, w, m1, m0, g, factor, dtype):
    M1, W1 = ro.muon_step(g, m0, w, LR, MU, True, WD, float(np.float32(factor)))
    close(m1, M1, 2 * U * (np.abs(MU * m0) + np.abs(M1)), "momentum")
    _, err = _bound(g + MU * M1, dtype)
    off = np.linalg.norm(got - W1)
    assert off <= LR * factor * err + (HALF[dtype] + 4 * U) * np.linalg.norm(W1), (off, factor)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,I", [(64, 256), (256, 64), (192, 128), (128, 128)])
def test_gate_up_and_down_by_themselves(H, I, dtype):
    """gate, up: H in, I out; down: I in, H out.  Each is the oracle's update of that matrix with (out / in)^0.5 where it gives out more."""
    b = _block(H, I, dtype)
    m = [np.zeros((b.E, H, I)), np.zeros((b.E, H, I)), np.zeros((b.E, I, H))]
    for step in range(2):
        print(f"update H={H} I={I} {dtype} step {step}", flush=True)
        _gradients(b, step)
        before = f64(b.w_gate_up), f64(b.w_down)
        g = f64(b.dw_gate_up), f64(b.dw_down)
        b.update(lr=0.05, mu=0.9, weight_decay=0.1, scale="fan", apart=True)
        after, mom = (f64(b.w_gate_up), f64(b.w_down)), [f64(t) for t in b.momentum]
        for e in range(b.E):
            for h, cols in enumerate((slice(0, I), slice(I, 2 * I))):
                _check(after[0][e][:, cols], before[0][e][:, cols], mom[0][h * b.E + e], m[h][e], g[0][e][:, cols], max(1.0, I / H) ** 0.5, dtype)
                m[h][e] = mom[0][h * b.E + e]
            _check(after[1][e], before[1][e], mom[1][e], m[2][e], g[1][e], max(1.0, H / I) ** 0.5, dtype)
            m[2][e] = mom[1][e]
    with pytest.raises(ValueError, match="apart"):
        b.update(lr=0.05)


@pytest.mark.parametrize("H,I", [(256, 64), (64, 256)])
def test_as_one_matrix(H, I):
    """[H, 2I] as stored; the factor is the caller's, 1 unless said otherwise, or from H in and 2I out."""
    for scale, factors in ((None, (1.0, 1.0)), (1.5, (1.5, 1.5)), ("fan", (max(1.0, 2 * I / H) ** 0.5, max(1.0, H / I) ** 0.5))):
        b = _block(H, I, "f32")
        _gradients(b, 5)
        before, g = (f64(b.w_gate_up), f64(b.w_down)), (f64(b.dw_gate_up), f64(b.dw_down))
        b.update(lr=0.05, mu=0.9, weight_decay=0.1, **({} if scale is None else dict(scale=scale)))
        for n, got, w0, g0, m in zip(range(2), (f64(b.w_gate_up), f64(b.w_down)), before, g, b.momentum):
            for e in range(b.E):
                _check(got[e], w0[e], f64(m)[e], np.zeros_like(w0[e]), g0[e], factors[n], "f32")
        with pytest.raises(ValueError, match="apart"):
            b.update(lr=0.05, apart=True)


def test_step_and_update_with_gate_and_up_apart():
    """A training step, its update, and the next step on the weights that it leaves."""
    T, H, I, E = 96, 128, 192, 8
    b = MoeBlock(T, H, I, E, 2, seed=1, scores=moe.make_scores("sigmoid", 4, 2))
    g = torch.Generator("cuda").manual_seed(0)
    x, dout, dz = (torch.randn(T, H, generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    for _ in range(2):
        b.step(x, dout, dz)
        before = b.w_gate_up.clone(), b.w_down.clone()
        b.update(lr=0.02, scale="fan", apart=True)
        for w, old in zip((b.w_gate_up, b.w_down), before):
            assert torch.isfinite(w).all() and not torch.equal(w, old)
        # singular values of the steps lie around lr times the factor, between 0.7 and 1.2 of it where they are not a small part of the whole
        for h in range(2):
            d = (b.w_gate_up[0, :, h * I:(h + 1) * I].float() - before[0][0, :, h * I:(h + 1) * I].float())
            assert torch.linalg.matrix_norm(d.double(), 2) <= 0.02 * (I / H) ** 0.5 * 1.25 + 2.0 ** -8 * torch.linalg.vector_norm(b.w_gate_up[0].float())
