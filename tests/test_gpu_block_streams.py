"""Every operator around the layer on a stream of its own: the inputs become right on that stream only, behind some milliseconds of work, so a
launch on any other stream would read what they held before."""
import pytest
import torch

import paper_2605_23764_amd as moe

pytestmark = pytest.mark.gpu

T, H, I, E, K = 300, 320, 128, 16, 3
BF, F32 = torch.bfloat16, torch.float32


def _new(*shape, dtype=BF):
    return torch.full(shape, float("nan") if dtype.is_floating_point else 1, dtype=dtype, device="cuda")


def _inputs(g):
    def normal(*shape, dtype=BF):
        return torch.randn(*shape, generator=g, device="cuda").to(dtype)
    logits = normal(T, E, dtype=F32)
    return dict(x=normal(T, H), v=normal(T, H), dy=normal(T, H), dres=normal(T, H), gamma=normal(H), beta=normal(H),
                rng=torch.tensor([7, 8], device="cuda"), logits=logits, idx=logits.topk(K, dim=1).indices.int(), w=logits.topk(K, dim=1).values.softmax(1),
                dw=normal(T, K, dtype=F32), mask=(torch.rand(T, generator=g, device="cuda") < 0.8), dloss=normal(1, dtype=F32),
                w1=normal(E, H, 2 * I) / 16, w2=normal(E, I, H) / 16)


def _norm(a, s):
    y, mean, rstd, ws = _new(T, H), _new(T, dtype=F32), _new(T, dtype=F32), moe.alloc_layer_norm_workspace(T, H)
    dx, dg, db = _new(T, H), _new(H), _new(H)
    moe.moe_layer_norm_forward(a["x"], a["gamma"], a["beta"], 1e-5, y, mean, rstd, stream=s)
    moe.moe_layer_norm_backward(a["dy"], a["x"], a["gamma"], mean, rstd, a["dres"], dx, dg, db, ws, stream=s)
    over = a["dy"]                                                       # in place: the column sums are a launch of their own, ahead
    moe.moe_layer_norm_backward(over, a["x"], a["gamma"], mean, rstd, None, over, dg, None, ws, stream=s)
    return y, mean, rstd, dx, dg, db, over


def _dropout(a, s):
    out, dv = _new(T, H), _new(T, H)
    moe.moe_dropout_add_forward(a["v"], a["x"], 0.3, a["rng"], out, stream=s)
    moe.moe_dropout_add_backward(a["dy"], 0.3, a["rng"], dv, stream=s)
    return out, dv


def _dropout_norm(a, s):
    z, y, mean, rstd, ws = _new(T, H), _new(T, H), _new(T, dtype=F32), _new(T, dtype=F32), moe.alloc_layer_norm_workspace(T, H)
    dz, dv, dg, db = _new(T, H), _new(T, H), _new(H), _new(H)
    moe.moe_dropout_add_layer_norm_forward(a["v"], a["x"], 0.3, a["rng"], a["gamma"], a["beta"], 1e-5, z, y, mean, rstd, stream=s)
    moe.moe_dropout_add_layer_norm_backward(a["dy"], z, a["gamma"], mean, rstd, a["dres"], 0.3, a["rng"], dz, dv, dg, db, ws, stream=s)
    return z, y, mean, rstd, dz, dv, dg, db


def _router(a, s):
    counts, prob, loss, dl = _new(E + 1, dtype=torch.int32), _new(E, dtype=F32), _new(1, dtype=F32), _new(T, E, dtype=F32)
    moe.moe_balance_forward(a["logits"], a["idx"], a["mask"], 0.1, counts, prob, loss, moe.alloc_balance_workspace(T, E), stream=s)
    moe.moe_router_backward(a["logits"], a["idx"], a["w"], a["dw"], a["mask"], 0.1, counts, a["dloss"], dl, stream=s)
    return counts, prob, loss, dl


def _experts(a, s):
    blocks = []
    for w in (a["w1"], a["w2"]):
        q, sc = moe.alloc_w4(*w.shape)
        moe.moe_quantize_w4(w, q, sc, stream=s)
        blocks += [q, sc]
    outs = []
    for t in (2, 40, 300):                                              # without a routing launch, with one, tiles
        shape = moe.make_shape(t, H, I, E, E, 0, K, BF)
        ws, out = moe.alloc_workspace(shape), _new(t, H)
        moe.moe_ffn_forward_w4(shape, a["x"][:t], a["logits"][:t], *blocks, out, None, ws, stream=s)
        outs += [out, ws]                                               # (the workspace too: it has to live until the stream is through)
    return *blocks, *outs[::2], *outs[1::2]


@pytest.mark.parametrize("calls,compared", [(_norm, 7), (_dropout, 2), (_dropout_norm, 8), (_router, 4), (_experts, 7)],
                         ids=["norm", "dropout", "dropout_norm", "router", "experts"])
@pytest.mark.parametrize("current", [False, True], ids=["argument", "current"])
def test_follows_its_stream(calls, compared, current):
    good, stale = (_inputs(torch.Generator("cuda").manual_seed(i)) for i in (1, 2))
    busy = torch.randn(4096, 4096, device="cuda")
    want = [t.clone() for t in calls({n: t.clone() for n, t in good.items()}, None)[:compared]]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(8):
            busy = (busy @ busy) * 1e-2
        for n, t in stale.items():
            t.copy_(good[n])
    if current:
        with torch.cuda.stream(s):
            kept = calls(stale, None)
    else:
        kept = calls(stale, s)
    s.synchronize()
    torch.cuda.synchronize()
    for i, (p, q) in enumerate(zip(kept[:compared], want)):
        assert torch.equal(p, q), i
