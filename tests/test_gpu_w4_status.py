"""moe_ffn_last_status behind a 4-bit layer, with and without a routing launch: what the workspace held before does not show."""
import pytest
import torch

import paper_2605_23764_amd as moe

pytestmark = pytest.mark.gpu

STATUS = 2                    # word of the workspace's header; MOE_ERR_SCHED_TIMEOUT is what a persistent launch may have left there
TIMEOUT = -5


@pytest.mark.parametrize("with_saved", [False, True], ids=["workspace", "saved"])
@pytest.mark.parametrize("T", [1, 16, 17])
def test_status_is_of_this_call(T, with_saved):
    shape = moe.make_shape(T, 128, 64, 8, 8, 0, 2, torch.bfloat16)
    g = torch.Generator("cuda").manual_seed(T)
    x = torch.randn(T, 128, generator=g, device="cuda").to(torch.bfloat16)
    logits = torch.randn(T, 8, generator=g, device="cuda")
    blocks = []
    for K, N in ((128, 128), (64, 128)):
        q, s = moe.alloc_w4(8, K, N)
        moe.moe_quantize_w4(torch.randn(8, K, N, generator=g, device="cuda") * K ** -0.5, q, s)
        blocks += [q, s]
    ws, out = moe.alloc_workspace(shape), torch.empty_like(x)
    saved = moe.alloc_saved(shape) if with_saved else None
    meta = moe.moe_ffn_debug_layout(shape)[0]
    for before in (TIMEOUT, -1):
        ws.fill_(255)
        ws[meta:meta + 16].view(torch.int32)[STATUS] = before
        torch.cuda.synchronize()
        assert moe.moe_ffn_last_status(shape, ws) == before
        moe.moe_ffn_forward_w4(shape, x, logits, *blocks, out, saved, ws)
        torch.cuda.synchronize()
        assert moe.moe_ffn_last_status(shape, ws) == 0
    assert not torch.isnan(out.float()).any()
