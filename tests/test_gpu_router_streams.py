"""Routing by scores, the router's projection and the orthogonal updates on streams of their own and beside each other; and the calls of the
largest sizes: more rows than a launch takes, offsets beyond 32 bits, many matrices of a few steps."""
import numpy as np
import pytest
import torch

import paper_2605_23764_amd as moe
from block_common import U, close
from oracle import router_oracle as ro

pytestmark = pytest.mark.gpu

T, H, I, E, K = 300, 320, 128, 16, 3
BF, F32 = torch.bfloat16, torch.float32


def _new(*shape, dtype=BF):
    return torch.full(shape, float("nan") if dtype.is_floating_point else 1, dtype=dtype, device="cuda")


def _inputs(seed):
    g = torch.Generator("cuda").manual_seed(seed)

    def normal(*shape, dtype=BF):
        return torch.randn(*shape, generator=g, device="cuda").to(dtype)
    return dict(x=normal(T, H), dy=normal(T, H), logits=normal(T, E, dtype=F32), bias=normal(E, dtype=F32) * 0.1, w=normal(H, E, dtype=F32),
                dlogits=normal(T, E, dtype=F32), dtopk=normal(T, K, dtype=F32), u=normal(3, 130, 200), m=normal(3, 130, 200, dtype=F32),
                w1=normal(E, H, 2 * I) / 16, w2=normal(E, I, H) / 16)


SCORES = [moe.make_scores("sigmoid", 4, 2, True, 2.5), moe.make_scores("softmax", 1, 1, False, 1.0)]


def _route(a, s):
    outs, kept = [], []
    for t in (5, T):                                                   # one launch, two
        for scores in SCORES:
            shape = moe.make_shape(t, H, I, E, E, 0, K, BF)
            saved, ws = moe.alloc_saved(shape, keep_xp=False), moe.alloc_workspace(shape)
            dl, bias = _new(t, E, dtype=F32), _new(E, dtype=F32)
            moe.moe_route_scores(shape, scores, a["logits"][:t], a["bias"], saved, ws, stream=s)
            moe.moe_route_scores_backward(scores, a["logits"][:t], saved.topk_idx, a["dtopk"][:t], a["dlogits"][:t], dl, stream=s)
            moe.moe_bias_update(saved.counts, 0.25, a["bias"], bias, stream=s)
            outs += [saved.topk_idx, saved.topk_w, saved.row_of, dl, bias]
            kept += [saved, ws]
    return outs, kept


def _project(a, s):
    ws = moe.alloc_router_project_workspace(T, H, E)
    logits, dx, dw = _new(T, E, dtype=F32), _new(T, H), _new(H, E, dtype=F32)
    moe.moe_router_project(a["x"], a["w"], logits, ws, stream=s)
    moe.moe_router_project_backward(a["dlogits"], a["x"], a["w"], a["dy"], dx, dw, ws, stream=s)
    return [logits, dx, dw], [ws]


def _updates(a, s):
    ws = moe.alloc_muon_workspace(3, 130, 200, BF)
    o, m, w = _new(3, 130, 200), _new(3, 130, 200, dtype=F32), _new(3, 130, 200)
    moe.moe_orthogonalize(a["u"], o, ws, stream=s)
    moe.moe_muon_step(a["u"], a["m"], a["u"], m, w, ws, 0.1, mu=0.9, weight_decay=0.1, stream=s)
    return [o, m, w], [ws]


def _experts(a, s):
    blocks = []
    for w in (a["w1"], a["w2"]):
        q, sc = moe.alloc_w4(*w.shape)
        moe.moe_quantize_w4(w, q, sc, stream=s)
        blocks += [q, sc]
    outs, kept = [], list(blocks)
    for t in (2, 40, T):
        shape = moe.make_shape(t, H, I, E, E, 0, K, BF)
        saved, ws, out = moe.alloc_saved(shape, keep_xp=False), moe.alloc_workspace(shape), _new(t, H)
        moe.moe_route_scores(shape, SCORES[0], a["logits"][:t], a["bias"], saved, ws, stream=s)
        moe.moe_dispatch_to_combine_w4(shape, a["x"][:t], *blocks, out, saved, ws, stream=s)
        outs.append(out)
        kept += [saved, ws]
    return outs, kept


CALLS = [_route, _project, _updates, _experts]


@pytest.mark.parametrize("calls", CALLS, ids=["route", "project", "updates", "experts"])
@pytest.mark.parametrize("current", [False, True], ids=["argument", "current"])
def test_follows_its_stream(calls, current):
    """The inputs become right on that stream only, behind some milliseconds of work."""
    good, stale = _inputs(1), _inputs(2)
    busy = torch.randn(4096, 4096, device="cuda")
    want = [t.clone() for t in calls(good, None)[0]]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(8):
            busy = (busy @ busy) * 1e-2
        for n, t in stale.items():
            t.copy_(good[n])
    if current:
        with torch.cuda.stream(s):
            got = calls(stale, None)
    else:
        got = calls(stale, s)
    s.synchronize()
    torch.cuda.synchronize()
    for i, (p, q) in enumerate(zip(got[0], want)):
        assert torch.equal(p, q), i


def test_beside_each_other():
    """All of them at once on four streams, each call with a workspace of its own, are what they are alone."""
    a = [_inputs(i) for i in range(4)]
    want = [[[t.clone() for t in calls(x, None)[0]] for calls in CALLS] for x in a]
    streams = [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    got = [[calls(x, s) for calls in CALLS] for x, s in zip(a, streams)]
    torch.cuda.synchronize()
    for mine, right in zip(got, want):
        for p, q in zip(mine, right):
            assert all(torch.equal(x, y) for x, y in zip(p[0], q))


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("t,e,k,G,top", [(12, 64, 6, 4, 2), (300, 64, 6, 4, 2), (300, 255, 8, 1, 1), (40, 256, 16, 8, 3)])
def test_scores_that_vanish(t, e, k, G, top, kind):
    """Scores of exactly zero beside others, and nothing but them: they tie, the lowest expert first, unless a bias tells them apart."""
    r = np.random.default_rng(t + e)
    L = np.where(r.random((t, e)) < 0.9, -1000.0, r.normal(size=(t, e))).astype(np.float32)
    L[0] = -1e30
    L[1, :] = np.where(np.arange(e) % 2, -3e38, -np.inf)
    L[2] = 0.0
    for bias in (None, np.where(np.arange(e) % 3, 0.0, 2.0 ** -20).astype(np.float32)):
        shape = moe.make_shape(t, 64, 64, e, e, 0, k, BF)
        saved, ws = moe.alloc_saved(shape, keep_xp=False), moe.alloc_workspace(shape)
        moe.moe_route_scores(shape, moe.make_scores(kind, G, top, True, 2.0), torch.from_numpy(L).cuda(), None if bias is None else torch.from_numpy(bias).cuda(),
                             saved, ws)
        idx, s = ro.select(L, kind, k, bias, G, top)
        np.testing.assert_array_equal(saved.topk_idx.cpu().numpy(), idx)
        w = ro.weights(s, idx, True, 2.0)
        close(saved.topk_w, w, U * w * 1.001 + 2.0 ** -148, "topk_w")


def test_more_rows_than_a_launch_of_dx():
    t, h, e = (1 << 21) + 300, 8, 3
    g = torch.Generator("cuda").manual_seed(0)
    d, w = torch.randn(t, e, generator=g, device="cuda"), torch.randn(h, e, generator=g, device="cuda")
    x, dres = (torch.randn(t, h, generator=g, device="cuda").to(BF) for _ in range(2))
    ws = moe.alloc_router_project_workspace(t, h, e)
    dx = _new(t, h)
    moe.moe_router_project_backward(d, x, w, dres, dx, None, ws)
    for a, b in ((0, 200), ((1 << 21) - 130, t)):
        part = _new(b - a, h)
        moe.moe_router_project_backward(d[a:b].clone(), x[a:b].clone(), w, dres[a:b].clone(), part, None, ws)
        assert torch.equal(dx[a:b], part)
    over = dres.clone()
    moe.moe_router_project_backward(d, x, w, over, over, None, ws)
    assert torch.equal(over, dx)


def test_as_many_tokens_as_there_are_numbers():
    """The most tokens that the limits allow, of one value and one expert: the last ones count as the first."""
    t = (1 << 31) - 129
    x, d = torch.zeros(t, 1, dtype=BF, device="cuda"), torch.zeros(t, 1, device="cuda")
    at = torch.tensor([0, 1 << 20, (1 << 30) + 7, t - 9000000, t - 1000, t - 1], device="cuda")
    x[at, 0] = torch.arange(1, 7, dtype=BF, device="cuda")
    d[at, 0] = torch.tensor([1.0, 0.5, 2.0, -3.0, 0.25, 4.0], device="cuda")
    w = torch.full((1, 1), 1.5, device="cuda")
    ws, dw = moe.alloc_router_project_workspace(t, 1, 1), _new(1, 1, dtype=F32)
    moe.moe_router_project_backward(d, x, w, None, None, dw, ws)
    assert dw.item() == 1.0 + 1.0 + 6.0 - 12.0 + 1.25 + 24.0
    dx = _new(t, 1)
    moe.moe_router_project_backward(d, x, w, None, dx, None, ws)
    assert torch.equal(dx[at, 0].float(), d[at, 0] * 1.5) and torch.count_nonzero(dx).item() == 6
    logits = d.fill_(-1.0)
    moe.moe_router_project(x, w, logits, ws)
    assert torch.equal(logits[at, 0], x[at, 0].float() * 1.5) and torch.count_nonzero(logits).item() == 6


@pytest.mark.parametrize("M,N", [(70, 100), (190, 70), (3, 250)])
def test_many_matrices_of_few_steps(M, N):
    """As many as there are compute units and a few more: whole tiles whose reductions are two to four steps long; each is what it is alone."""
    n = 270
    u = torch.randn(n, M, N, generator=torch.Generator("cuda").manual_seed(M), device="cuda").to(BF)
    out, one = torch.empty_like(u), torch.empty(1, M, N, dtype=BF, device="cuda")
    ws = moe.alloc_muon_workspace(n, M, N, BF)
    moe.moe_orthogonalize(u, out, ws)
    for e in (0, 1, 128, 255, 256, n - 1):
        moe.moe_orthogonalize(u[e:e + 1].clone(), one, ws)
        assert torch.equal(out[e], one[0]), e
