"""One workspace, as large as the largest call asks for, through smaller calls: they are taken, give the same bits as with one of their own, and
leave what lies behind it alone."""
import pytest
import torch

import paper_2605_23764_amd as moe

pytestmark = pytest.mark.gpu


def _guarded(size):
    whole = torch.full((size + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    return whole[:size], whole[size:]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("largest,H,E,smaller", [(37, 7168, 256, (36, 33, 1)), (3000, 7168, 256, (2048, 1025, 129, 36)), (5500, 1024, 128, (2100, 260, 64)),
                                                 (900, 1001, 24, (640, 641, 65, 3))])
def test_router_project(largest, H, E, smaller, dtype):
    g = torch.Generator("cuda").manual_seed(H)
    x, dres = (torch.randn(largest, H, generator=g, device="cuda").to(dtype) for _ in range(2))
    w, d = torch.randn(H, E, generator=g, device="cuda"), torch.randn(largest, E, generator=g, device="cuda")
    ws, behind = _guarded(moe.moe_router_project_workspace_bytes(largest, H, E))
    for T in (largest, *smaller):
        print(f"project T={T} of {largest}, H={H} E={E} {dtype}", flush=True)
        results = []
        for space in (moe.alloc_router_project_workspace(T, H, E), ws):
            logits, dx, dw = torch.empty(T, E, device="cuda"), torch.empty(T, H, dtype=dtype, device="cuda"), torch.empty(H, E, device="cuda")
            moe.moe_router_project(x[:T], w, logits, space)
            moe.moe_router_project_backward(d[:T], x[:T], w, dres[:T], dx, dw, space)
            results.append((logits, dx, dw))
        assert all(torch.equal(a, b) for a, b in zip(*results))
        assert (behind == 0xA5).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_muon(dtype):
    """16400 matrices go in groups of 8200, 16384 in one."""
    M, N = 8, 40
    u = torch.randn(16400, M, N, generator=torch.Generator("cuda").manual_seed(0), device="cuda").to(dtype)
    ws, behind = _guarded(moe.moe_muon_workspace_bytes(16400, M, N, dtype))
    for B in (16400, 16384, 8201, 3):
        print(f"orthogonalize {B} of 16400 x {M} x {N} {dtype}", flush=True)
        results = []
        for space in (moe.alloc_muon_workspace(B, M, N, dtype), ws):
            out = torch.empty_like(u[:B])
            moe.moe_orthogonalize(u[:B], out, space)
            results.append(out)
        assert torch.equal(*results) and torch.isfinite(results[0]).all()
        assert (behind == 0xA5).all()
