"""A single launch behind a routing that has left its counters and task tables out: whatever the workspace holds, it computes nothing, leaves the output
as it was and says so; with them the next one is right."""
import pytest
import torch

import paper_2605_23764_amd as moe

pytestmark = pytest.mark.gpu

# tokens and type: weight streams (up to 64 tokens in bf16; routing by scores in one launch, in two), tile tasks, with a permuted copy and without
CASES = [(5, torch.bfloat16, False), (40, torch.bfloat16, True), (700, torch.bfloat16, False), (700, torch.bfloat16, True), (30, torch.float32, True),
         (300, torch.float32, False)]


def _layer(T, dtype, keep_xp):
    H, I, E, El, base, k = 128, 64, 16, 10, 3, 3
    g = torch.Generator("cuda").manual_seed(T)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)
    shape = moe.make_shape(T, H, I, E, El, base, k, dtype)
    return shape, normal(T, H), normal(El, H, 2 * I, scale=H ** -0.5), normal(El, I, H, scale=I ** -0.5), torch.randn(T, E, generator=g, device="cuda"), \
        moe.alloc_saved(shape, store_h1=True, keep_xp=keep_xp)


def _route(how, shape, x, w1, w2, logits, saved, ws, mode):
    if how == "scores":
        moe.moe_route_scores(shape, moe.make_scores("softmax"), logits, None, saved, ws, mode)
    else:
        moe.moe_ffn_forward(shape, x, logits, w1, w2, torch.empty_like(x), saved, ws, mode)


@pytest.mark.parametrize("T,dtype,keep_xp", CASES)
@pytest.mark.parametrize("held", ["ones", "zeros", "an earlier routing's"])
@pytest.mark.parametrize("how", ["scores", "forward"])
def test_single_launch_without_tables(T, dtype, keep_xp, held, how):
    print(f"T={T} {dtype} Xp {keep_xp}, {held} in the workspace, {how}", flush=True)
    shape, x, w1, w2, logits, saved = _layer(T, dtype, keep_xp)
    ws, out = moe.alloc_workspace(shape), torch.full_like(x, 7.0)
    ws.fill_(255 if held == "ones" else 0)
    if held == "an earlier routing's":
        moe.moe_route(shape, torch.roll(logits, 1, 0).contiguous(), saved, ws)
    _route(how, shape, x, w1, w2, logits, saved, ws, moe.MODE_SERIALIZED)
    for t in (saved.A, saved.Yp):
        t.fill_(3.0)
    moe.moe_dispatch_to_combine(shape, x, w1, w2, out, saved, ws, moe.MODE_PERSISTENT)
    torch.cuda.synchronize()
    assert moe.moe_ffn_last_status(shape, ws) == -7 and "without" in moe.moe_status_string(-7)
    assert (out == 7.0).all() and (saved.A == 3.0).all() and (saved.Yp == 3.0).all()
    # the serialized mode runs on that routing, and a routing for the single launch clears the word
    want = torch.empty_like(x)
    moe.moe_dispatch_to_combine(shape, x, w1, w2, want, saved, ws, moe.MODE_SERIALIZED)
    if how == "scores":
        _route(how, shape, x, w1, w2, logits, saved, ws, moe.MODE_PERSISTENT)
    else:
        moe.moe_route(shape, logits, saved, ws)
    moe.moe_dispatch_to_combine(shape, x, w1, w2, out, saved, ws, moe.MODE_PERSISTENT)
    torch.cuda.synchronize()
    assert moe.moe_ffn_last_status(shape, ws) == 0
    assert torch.equal(out, want) and torch.isfinite(out).all()
