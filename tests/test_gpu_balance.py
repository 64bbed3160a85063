"""Balance loss, counts and the router's backward on the GPU, against the fp64 oracle: every number of lanes per token, odd expert counts,
one workgroup and many, masks up to all tokens, -inf logits, missing parts."""
import numpy as np
import pytest
import torch

import paper_2605_23764_amd as moe
from block_common import U, close, f64
from oracle import block_oracle as bo

pytestmark = pytest.mark.gpu

# lanes per token 1, 2, 4, 8, 16, 32, 64; E not a multiple of 4; one workgroup, two launches
SHAPES = [(1, 1, 1), (1, 256, 8), (5, 3, 3), (64, 4, 1), (65, 8, 2), (200, 7, 7), (1000, 16, 4), (333, 24, 3), (4097, 60, 6), (777, 64, 8),
          (500, 127, 5), (300, 128, 16), (900, 250, 8), (3001, 256, 8), (20000, 33, 2), (20003, 256, 8), (70000, 9, 3), (128, 256, 8), (129, 256, 8), (8192, 4, 1), (8193, 3, 2)]


def _inputs(T, E, k, seed, masked=None, hole=0.0):
    """masked: share of tokens off; hole: share of logits at -inf beyond the first k + 1 experts."""
    r = np.random.default_rng(seed)
    logits = (2.0 * r.normal(size=(T, E)) + r.normal(size=E)).astype(np.float32)
    if hole:
        logits[:, k + 1:][r.random((T, max(0, E - k - 1))) < hole] = -np.inf
    idx = np.argsort(-logits, axis=1, kind="stable")[:, :k].astype(np.int32)
    sel = np.take_along_axis(logits, idx.astype(np.int64), 1)
    w = np.exp(sel - sel[:, :1])
    w = (w / w.sum(1, keepdims=True)).astype(np.float32)
    dw = r.normal(size=(T, k)).astype(np.float32)
    mask = None if masked is None else (r.random(T) >= masked).astype(np.uint8)
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    return (logits, idx, w, dw, mask), tuple(dev(a) for a in (logits, idx, w, dw, mask))


def _forward(logits, idx, mask, coef):
    T, E = logits.shape
    counts = torch.full((E + 1,), -7, dtype=torch.int32, device="cuda")
    prob, loss = torch.full((E,), float("nan"), device="cuda"), torch.full((1,), float("nan"), device="cuda")
    ws = torch.full((moe.moe_balance_workspace_bytes(T, E),), 255, dtype=torch.uint8, device="cuda")
    moe.moe_balance_forward(logits, idx, mask, coef, counts, prob, loss, ws)
    return counts, prob, loss


def _q_bound(logits):
    """(q, relative bound of its error): the exponent's argument is off by its own rounding, exp by two steps, the sum by 6 + 4, the
    reciprocal and the product by one each."""
    l = logits.astype(np.float64)
    q = bo.router_probabilities(l)
    span = np.where(np.isfinite(l), l.max(1, keepdims=True) - l, 0.0)
    span[~np.isfinite(span)] = 0.0
    e = U * (span + 4 + 12) + U * (q * span).sum(1, keepdims=True)
    return q, 2 * e


@pytest.mark.parametrize("masked", [None, 0.3], ids=["all", "masked"])
@pytest.mark.parametrize("T,E,k", SHAPES)
def test_balance_and_router_backward(T, E, k, masked):
    print(f"balance T={T} E={E} k={k} masked={masked}", flush=True)
    coef, dloss = 0.02, 1.75
    (L, I, W, D, M), (logits, idx, w, dw, mask) = _inputs(T, E, k, 17 * E + T, masked)
    counts, prob, loss = _forward(logits, idx, mask, coef)
    c, n, ps, ls = bo.balance(L.astype(np.float64), I, M, coef)
    assert counts.cpu().tolist() == [*c.tolist(), n]
    on = np.ones(T, bool) if M is None else M != 0
    q, e_q = _q_bound(L)
    # sums over tokens: a lane's own one after the other, at most T / 128 (or all of up to 64), then 6 + 8 + 32 + 4
    steps = (T / 128 + 64 + 50) * U
    e_p = (q * e_q)[on].sum(0) + steps * ps
    close(prob, ps, e_p, "prob_sum")
    f = c / max(1, k * n)
    close(loss, np.array([ls]), coef * E * (f * e_p).sum() / max(1, n) + 24 * U * ls, "loss")
    dl = torch.tensor([dloss], device="cuda")
    for use_w, use_c in ((True, True), (True, False), (False, True), (False, False)):
        got = torch.full_like(logits, float("nan"))
        moe.moe_router_backward(logits, idx, w if use_w else None, dw if use_w else None, mask, coef, counts if use_c else None, dl, got)
        want = bo.router_backward(L.astype(np.float64), I, W.astype(np.float64) if use_w else None, D.astype(np.float64), M, coef,
                                  c if use_c else None, n, dloss)
        tol = np.zeros((T, E))
        if use_c and n:
            a = dloss * coef * E / n
            fq = (q * f).sum(1, keepdims=True)
            tol += a * q * (e_q * (f + fq) + (f * q * e_q).sum(1, keepdims=True) + 16 * U * (f + fq)) * on[:, None]
        if use_w:
            dot = np.abs(W * D).sum(1, keepdims=True)
            share = np.zeros((T, E))
            np.put_along_axis(share, I.astype(np.int64), W * (np.abs(D) + dot) * 24 * U, 1)
            tol += share
        close(got, want, tol + 2 * U * np.abs(want), f"dlogits {use_w} {use_c}")
        if use_w and use_c:
            same = logits.clone()
            moe.moe_router_backward(same, idx, w, dw, mask, coef, counts, dl, same)
            assert torch.equal(same, got)


def test_no_token_counts():
    (L, I, W, D, _), (logits, idx, w, dw, _) = _inputs(200, 16, 3, 1)
    mask = torch.zeros(200, dtype=torch.bool, device="cuda")
    counts, prob, loss = _forward(logits, idx, mask, 0.1)
    assert (counts == 0).all() and (prob == 0).all() and loss.item() == 0.0
    got, want = torch.empty_like(logits), torch.empty_like(logits)
    moe.moe_router_backward(logits, idx, w, dw, mask, 0.1, counts, None, got)
    moe.moe_router_backward(logits, idx, w, dw, None, 0.1, None, None, want)
    assert torch.equal(got, want)
    empty = torch.empty(0, 16, device="cuda")
    counts, prob, loss = _forward(empty, torch.empty(0, 3, dtype=torch.int32, device="cuda"), None, 0.1)
    assert (counts == 0).all() and (prob == 0).all() and loss.item() == 0.0


def test_masked_experts_and_rows():
    """-inf logits have probability and gradient 0; a row of nothing else has none at all and spoils no other; ids outside are left out."""
    (L, I, W, D, _), (logits, idx, w, dw, _) = _inputs(300, 32, 4, 2, hole=0.6)
    c, n, ps, ls = bo.balance(L.astype(np.float64), I, None, 0.1)
    counts, prob, loss = _forward(logits, idx, None, 0.1)
    q, e_q = _q_bound(L)
    close(prob, ps, (q * e_q).sum(0) + 120 * U * ps, "prob_sum")
    d = torch.empty_like(logits)
    moe.moe_router_backward(logits, idx, None, None, None, 0.1, counts, None, d)
    assert (d[torch.isinf(logits)] == 0).all() and not torch.isnan(d).any()
    logits[7] = float("-inf")
    idx[7] = -1
    idx[9, 1], idx[11, 0] = 32, -5
    counts, prob, loss = _forward(logits, idx, None, 0.1)
    L, I = logits.cpu().numpy(), idx.cpu().numpy()
    c, n, ps, _ = bo.balance(L.astype(np.float64), I, None, 0.1)
    assert counts.cpu().tolist() == [*c.tolist(), n] and n == 300
    close(prob, ps, (q * e_q).sum(0) + 120 * U * ps, "prob_sum")
    moe.moe_router_backward(logits, idx, w, dw, None, 0.1, counts, None, d)
    assert (d[7] == 0).all() and not torch.isnan(d).any()


def test_same_bits_again_and_nan_is_told():
    _, (logits, idx, w, dw, _) = _inputs(9000, 256, 8, 3)
    first = _forward(logits, idx, None, 0.1)
    assert all(torch.equal(a, b) for a, b in zip(first, _forward(logits, idx, None, 0.1)))
    logits[4000, 17] = float("nan")
    counts, prob, loss = _forward(logits, idx, None, 0.1)
    assert torch.equal(counts, first[0]) and torch.isnan(prob).all() and torch.isnan(loss).all()


def test_replays_from_a_graph():
    _, (logits, idx, w, dw, mask) = _inputs(3000, 64, 6, 4, masked=0.2)
    T, E = logits.shape
    counts, prob, loss = torch.empty(E + 1, dtype=torch.int32, device="cuda"), torch.empty(E, device="cuda"), torch.empty(1, device="cuda")
    d, ws = torch.empty_like(logits), moe.alloc_balance_workspace(T, E)

    def step():
        moe.moe_balance_forward(logits, idx, mask, 0.1, counts, prob, loss, ws)
        moe.moe_router_backward(logits, idx, w, dw, mask, 0.1, counts, None, d)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for seed in (5, 6, 5):
        _, (l, i, _, x, m) = _inputs(3000, 64, 6, seed, masked=0.5)
        logits.copy_(l), idx.copy_(i), dw.copy_(x), mask.copy_(m)
        for t in (counts, prob, loss, d):
            t.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (counts, prob, loss, d)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (counts, prob, loss, d)))


def test_counts_of_the_router_itself():
    """On what moe_route selects: the counts of the local experts are the layer's own."""
    T, E, k = 500, 24, 3
    shape = moe.make_shape(T, 64, 64, E, 10, 6, k, torch.float32)
    logits = torch.randn(T, E, generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    saved, ws = moe.alloc_saved(shape), moe.alloc_workspace(shape)
    moe.moe_route(shape, logits, saved, ws)
    counts, _, _ = _forward(logits, saved.topk_idx, None, 0.1)
    assert torch.equal(counts[6:16], saved.counts) and counts[:E].sum().item() == T * k
