"""The block's update of its experts: the factor from what a matrix takes in and gives out."""
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
