"""Workspace of the layer norm's backward: as much as its partial sums take, which are at most 256 rows of 2 H fp32, and nothing behind it
is touched."""
import pytest
import torch

import paper_2605_23764_amd as moe


@pytest.mark.parametrize("T,H", [(1, 8), (255, 1001), (256, 64), (257, 64), (513, 7168), (8192, 7168), (2 ** 31 - 1, 1)])
def test_bytes(T, H):
    assert moe.moe_layer_norm_workspace_bytes(T, H) == min(T, 256) * 2 * H * 4


@pytest.mark.gpu
@pytest.mark.parametrize("T,H", [(5000, 1001), (5000, 64), (40000, 72), (2000, 7168), (300, 8200), (900, 256)])
def test_nothing_behind_it(T, H):
    print(f"workspace T={T} H={H}", flush=True)
    g = torch.Generator("cuda").manual_seed(H)
    x, dy = (torch.randn(T, H, generator=g, device="cuda") for _ in range(2))
    y, mean, rstd = torch.empty_like(x), torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    moe.moe_layer_norm_forward(x, None, None, 1e-5, y, mean, rstd)
    n = moe.moe_layer_norm_workspace_bytes(T, H)
    whole = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    dx, dg, db = torch.empty_like(x), torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
    moe.moe_layer_norm_backward(dy, x, None, mean, rstd, None, dx, dg, db, whole[:n])
    assert (whole[n:] == 0xA5).all()
    # the sums of many terms: an fp32 step per term, on both sides
    tol = 2 * (T + 1100) * 2.0 ** -24
    d, xh = dy.double(), (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    assert ((dg - (d * xh).sum(0)).abs() <= tol * (d * xh).abs().sum(0) + 1e-6).all()
    assert ((db - d.sum(0)).abs() <= tol * d.abs().sum(0)).all()
