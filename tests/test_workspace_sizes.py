"""Workspaces of the largest call serve every smaller one: their sizes never fall, at the borders of splits and groups neither (CPU only)."""
import pytest
import torch

import paper_2605_23764_amd as moe


def _around(points, most):
    return sorted({v for p in points for v in range(p - 2, p + 3) if 1 <= v <= most})


# every T up to 700, then where the tiles of 128 rows and the steps of 64 change
TOKENS = sorted({*range(1, 700), *_around([128 * i for i in range(5, 130)], 1 << 20), *_around([1 << i for i in range(10, 21)], 1 << 20),
                 *_around([3 << i for i in range(9, 19)], 1 << 20)})


@pytest.mark.parametrize("H,E", [(1, 1), (33, 5), (96, 24), (1001, 60), (2048, 64), (4096, 128), (7168, 256), (5000, 3), (262144, 256), (320, 160)])
def test_router_project(H, E):
    taken = [T for T in TOKENS if -(-T // 128) * -(-max(H, E) // 64) < 1 << 24]      # the limit of a launch
    sizes = [moe.moe_router_project_workspace_bytes(T, H, E) for T in [0, *taken]]
    assert sizes == sorted(sizes)
    # two workgroups to each of 256 CUs, of 128 x 128 sums at most, or as many splits of dW
    assert sizes[-1] <= 2 * 256 * 128 * 128 * 4 + 256 * H * E * 4


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M,N", [(1, 1), (64, 64), (200, 330), (704, 1088), (2816, 2048), (7168, 4096), (4096, 7168), (16384, 32768), (30000, 30000)])
def test_muon(M, N, dtype):
    counts = sorted({*range(0, 400), *_around([1 << i for i in range(9, 18)], 1 << 20)})
    sizes = [moe.moe_muon_workspace_bytes(B, M, N, dtype) for B in counts]
    assert sizes == sorted(sizes)
    assert sizes[-1] <= max(sizes[1], 5 << 30)                       # that of a group, or of a matrix that is larger
    assert sizes == [moe.moe_muon_workspace_bytes(B, N, M, dtype) for B in counts]
