"""Routing by scores on the GPU, against the fp64 oracle: selections and tables to the bit, weights and gradients to their roundings; one
launch and two, every number of experts per lane, groups that straddle lanes, holes, ties, odd counts."""
import numpy as np
import pytest
import torch

import oracle
import paper_2605_23764_amd as moe
from block_common import U, close, f64
from oracle import router_oracle as ro

pytestmark = pytest.mark.gpu

# T, E, k, n_group, topk_group, E_local, base: up to 64 tokens one launch; a lane has 1, 2, 4, 8, 16 experts; groups of one, of odd sizes,
# that begin inside a lane
SHAPES = [(1, 256, 8, 8, 4, 32, 64), (1, 1, 1, 1, 1, 1, 0), (3, 8, 2, 1, 1, 8, 0), (5, 15, 4, 15, 6, 7, 8), (33, 60, 6, 4, 2, 20, 40), (64, 256, 16, 16, 2, 256, 0),
          (64, 24, 3, 3, 1, 10, 6), (65, 24, 8, 1, 1, 24, 0), (200, 60, 5, 12, 3, 60, 0), (100, 100, 7, 10, 5, 33, 50), (300, 250, 8, 10, 4, 100, 150),
          (777, 16, 1, 1, 1, 4, 12), (1000, 256, 8, 8, 4, 32, 0), (2050, 128, 6, 1, 1, 16, 16), (513, 64, 16, 8, 2, 8, 0), (40, 255, 8, 1, 1, 255, 0)]


def _logits(T, E, seed):
    r = np.random.default_rng(seed)
    return (1.5 * r.normal(size=(T, E)) + 0.5 * r.normal(size=E)).astype(np.float32), r


def _route(logits, scores, bias, k, E_local, base, dtype=torch.bfloat16, mode=moe.MODE_SERIALIZED):
    T, E = logits.shape
    shape = moe.make_shape(T, 64, 64, E, E_local, base, k, dtype)
    saved, ws = moe.alloc_saved(shape, keep_xp=False), moe.alloc_workspace(shape)
    for t in (saved.topk_idx, saved.counts, saved.offsets, saved.row_of, saved.token_of, saved.slot_of):
        t.fill_(-7)
    saved.topk_w.fill_(float("nan"))
    ws.fill_(255)
    moe.moe_route_scores(shape, scores, logits, bias, saved, ws, mode)
    return shape, saved, ws


def _check_tables(saved, idx, E_local, base):
    p = dict(zip(("counts", "offsets", "row_of", "token_of", "slot_of"), oracle.local_permutation(idx, base, E_local)))
    R = int(p["offsets"][-1])
    for n in ("counts", "offsets", "row_of"):
        np.testing.assert_array_equal(getattr(saved, n).cpu().numpy(), p[n], err_msg=n)
    for n in ("token_of", "slot_of"):
        np.testing.assert_array_equal(getattr(saved, n).cpu().numpy()[:R], p[n], err_msg=n)
        assert (getattr(saved, n)[R:] == -7).all(), n                # rows behind the last are left as they were


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renorm", [True, False], ids=["renorm", "plain"])
@pytest.mark.parametrize("T,E,k,G,top,El,base", SHAPES)
def test_selection_tables_weights_and_gradient(T, E, k, G, top, El, base, kind, renorm):
    print(f"route_scores T={T} E={E} k={k} groups={G}/{top} local={El}+{base} {kind} renorm={renorm}", flush=True)
    L, r = _logits(T, E, 7 * T + E)
    bias = None if E % 2 == 0 and T % 2 else (0.2 * r.normal(size=E)).astype(np.float32)
    scores = moe.make_scores(kind, G, top, renorm, 2.5)
    logits = torch.from_numpy(L).cuda()
    dev_bias = None if bias is None else torch.from_numpy(bias).cuda()
    idx, s = ro.select(L, kind, k, bias, G, top)
    for dtype, mode in ((torch.bfloat16, moe.MODE_SERIALIZED), (torch.float32, moe.MODE_SERIALIZED), (torch.bfloat16, moe.MODE_PERSISTENT)):
        shape, saved, ws = _route(logits, scores, dev_bias, k, El, base, dtype, mode)
        np.testing.assert_array_equal(saved.topk_idx.cpu().numpy(), idx)
        _check_tables(saved, idx, El, base)
        w = ro.weights(s, idx, renorm, 2.5)
        close(saved.topk_w, w, U * w * 1.001, "topk_w")             # 64 bits, rounded once
    # gradient: the slots in 64 bits and rounded; in 32: added to dadd, and for a softmax as it is, over all E, an exponential of an
    # argument off by its own rounding (2 steps), a sum (6 + 4 terms' worth), the product, the difference
    dw, dadd = (r.normal(size=n).astype(np.float32) for n in ((T, k), (T, E)))
    dev = [torch.from_numpy(a).cuda() for a in (dw, dadd)]
    part = ro.weights_backward(L.astype(np.float64), kind, idx, dw.astype(np.float64), renorm, float(np.float32(2.5)))
    tol = U * np.abs(part) * 2
    # the oracle's own: where the definition's terms cancel (a renormalised softmax, at the experts that were not selected), its up to 16
    # terms of at most 2.5 |dw| leave roundings of 2^-53 each, with those of the terms themselves 8 to a term
    tol += 16 * 8 * 2.0 ** -53 * 2.5 * np.abs(dw).max()
    if kind == "softmax" and not renorm:
        span = L.astype(np.float64).max(1, keepdims=True) - L
        e = U * (span + 20) + U * (s * (span + 20)).sum(1, keepdims=True)
        d = np.abs(2.5 * (np.take_along_axis(s, idx, 1) * dw).sum(1, keepdims=True))
        ds = 2.5 * (np.take_along_axis(s * e, idx, 1) * np.abs(dw)).sum(1, keepdims=True)
        tol = tol + s * d * (2 * e + 4 * U) + s * ds
        np.put_along_axis(tol, idx, np.take_along_axis(tol, idx, 1) + 2.5 * np.take_along_axis(s * e, idx, 1) * np.abs(dw) + 2 * U * 2.5 * np.take_along_axis(s, idx, 1) * np.abs(dw), 1)
    for add in (None, dev[1]):
        got = torch.full((T, E), float("nan"), device="cuda")
        moe.moe_route_scores_backward(scores, logits, saved.topk_idx, dev[0], add, got)
        want = part if add is None else part + dadd
        close(got, want, tol + 2 * U * (np.abs(part) + (0 if add is None else np.abs(dadd))) + 1e-45, f"dlogits, dadd {add is not None}")
        for over in ("logits", "dadd"):                             # outputs over inputs
            same = (logits if over == "logits" else dev[1]).clone()
            if over == "dadd" and add is None:
                continue
            moe.moe_route_scores_backward(scores, same if over == "logits" else logits, saved.topk_idx, dev[0], same if over == "dadd" else add, same)
            assert torch.equal(same, got), over


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("E,G,top,k", [(256, 2, 1, 16), (256, 4, 3, 8), (256, 16, 5, 8), (160, 8, 2, 8), (128, 2, 1, 5), (128, 8, 8, 6), (96, 6, 2, 8), (64, 2, 2, 6),
                                       (64, 16, 3, 4), (48, 4, 1, 12), (32, 16, 4, 8), (32, 4, 2, 1), (24, 2, 1, 3), (16, 16, 7, 7), (16, 4, 3, 5), (8, 2, 1, 4)])
def test_groups_of_every_width(E, G, top, k, kind):
    """Groups of whole lanes, one to sixteen of them, of more, of no power of two, that end inside a lane; few tokens and many; holes, ties of
    groups and of keys."""
    r = np.random.default_rng(E + G)
    bias = (r.integers(-2, 3, size=E) / 8).astype(np.float32)
    for T in (1, 16, 37, 200):
        L = (2 * r.normal(size=(T, E))).astype(np.float32)
        L[r.random((T, E)) < 0.2] = -np.inf
        L[::3] = np.round(L[::3])                                    # ties
        if T > 20:
            L[5] = 0.0
            L[6, : E // G] = -np.inf
            L[7, E // G:] = np.nan
            L[8] = -np.inf
        for b in (None, bias):
            _, saved, _ = _route(torch.from_numpy(L).cuda(), moe.make_scores(kind, G, top, True, 1.0), None if b is None else torch.from_numpy(b).cuda(), k, E, 0)
            idx, s = ro.select(L, kind, k, b, G, top)
            got = saved.topk_idx.cpu().numpy()
            # Two groups' sums that are equal as real numbers (s + 1/8 and s - 1/8 against s and s) are not after roundings, the oracle's neither.
            # Keys below 2 are rounded to 44 bits behind the point's first, off by 2^-45 at most, a sum of two of them below 4 by another 2^-44:
            # two groups are in doubt, and only then, within 2 (2 * 2^-45 + 2^-44) = 2^-42.
            for t in np.flatnonzero((got != idx).any(1)):
                key = np.where(np.isnan(L[t]) | (L[t] == -np.inf), -np.inf, s[t] + (0.0 if b is None else b.astype(np.float64)))
                two = np.sort(key.reshape(G, -1), axis=1)[:, ::-1][:, :2]
                value = two[:, 0] + np.where(two[:, 1:].max(axis=1, initial=-np.inf) > -np.inf, two[:, 1:].max(axis=1, initial=-np.inf), 0.0)
                order = np.sort(value)[::-1]
                assert order[top - 1] - order[top] <= 2.0 ** -42, (T, t)
                stay = set(got[t] // (E // G))
                assert all(value[g] >= order[top - 1] - 2.0 ** -42 for g in stay) and (np.diff(key[got[t]]) <= 0).all(), (T, t)
                idx[t] = got[t]
            w = ro.weights(s, idx, True, 1.0)
            close(saved.topk_w, w, U * w * 1.001 + 2.0 ** -149, "topk_w")


def test_keys_that_fp32_cannot_tell_apart():
    """Biased scores that differ by less than a rounding to fp32: the order is the definition's."""
    T, E, k = 500, 64, 6
    r = np.random.default_rng(1)
    L = (0.3 * r.normal(size=(T, E))).astype(np.float32)
    s = ro.scores(L[:1], "sigmoid")[0]
    bias = (1.0 - s).astype(np.float32)                             # token 0: every key is 1 up to roundings of the bias
    L[1:] = np.nextafter(L[0], np.where(r.random((T - 1, E)) < 0.5, np.inf, -np.inf).astype(np.float32))
    for T1 in (50, T):
        shape, saved, _ = _route(torch.from_numpy(L[:T1]).cuda(), moe.make_scores("sigmoid"), torch.from_numpy(bias).cuda(), k, E, 0)
        idx, _ = ro.select(L[:T1], "sigmoid", k, bias)
        np.testing.assert_array_equal(saved.topk_idx.cpu().numpy(), idx)


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("T", [40, 400])
def test_holes_ties_and_extremes(T, kind):
    E, k, G, top = 32, 5, 4, 2
    r = np.random.default_rng(T)
    L = r.integers(-2, 3, size=(T, E)).astype(np.float32)           # ties everywhere
    L[r.random((T, E)) < 0.3] = -np.inf
    L[3] = -np.inf
    L[5, :] = np.nan
    L[7, ::3] = np.inf
    L[9, 1:] = -np.inf
    L[11] = -200.0                                                  # scores that vanish in fp32
    L[13] = 3e38
    L[15, 4] = -0.0
    bias = r.integers(-1, 2, size=E).astype(np.float32)
    bias[6], bias[9], bias[10] = np.nan, np.inf, -np.inf
    for b in (None, bias):
        for renorm in (True, False):
            scores = moe.make_scores(kind, G, top, renorm, 1.5)
            logits, db = torch.from_numpy(L).cuda(), None if b is None else torch.from_numpy(b).cuda()
            _, saved, _ = _route(logits, scores, db, k, 20, 5)
            idx, s = ro.select(L, kind, k, b, G, top)
            np.testing.assert_array_equal(saved.topk_idx.cpu().numpy(), idx)
            _check_tables(saved, idx, 20, 5)
            w = ro.weights(s, idx, renorm, 1.5)
            close(saved.topk_w, w, U * w * 1.001 + 1.5 * 2.0 ** -149, "topk_w")
            dw = r.normal(size=(T, k)).astype(np.float32)
            got = torch.full((T, E), float("nan"), device="cuda")
            moe.moe_route_scores_backward(scores, logits, saved.topk_idx, torch.from_numpy(dw).cuda(), None, got)
            got = f64(got)
            assert np.isfinite(got).all()
            assert (got[~(L > -np.inf)] == 0).all() and (got[[3, 5]] == 0).all()
            fine = np.isfinite(L).any(1) & ~np.isinf(np.where(L == -np.inf, 0, L)).any(1)
            want = ro.weights_backward(L[fine].astype(np.float64), kind, idx[fine], dw[fine].astype(np.float64), renorm, 1.5)
            assert np.abs(got[fine] - want).max() <= 40 * U * np.abs(dw).max() * 1.5


def test_ids_outside_have_no_part():
    L, r = _logits(70, 24, 5)
    for kind in ("sigmoid", "softmax"):
        for renorm in (True, False):
            scores = moe.make_scores(kind, 1, 1, renorm, 1.0)
            idx, _ = ro.select(L, kind, 4)
            idx[3, 1], idx[9, 0], idx[11] = -1, 24, -5
            dw = r.normal(size=(70, 4)).astype(np.float32)
            got = torch.full((70, 24), float("nan"), device="cuda")
            moe.moe_route_scores_backward(scores, torch.from_numpy(L).cuda(), torch.from_numpy(idx.astype(np.int32)).cuda(), torch.from_numpy(dw).cuda(), None, got)
            want = ro.weights_backward(L.astype(np.float64), kind, idx, dw.astype(np.float64), renorm, 1.0)
            assert np.abs(f64(got) - want).max() <= 40 * U * np.abs(dw).max()
            assert (got[11] == 0).all()


@pytest.mark.parametrize("E", [1, 7, 64, 65, 256])
def test_bias_update(E):
    r = np.random.default_rng(E)
    counts = r.integers(0, 50, size=E + 1).astype(np.int32)
    counts[-1] = 123456                                             # moe_balance_forward's last word: not a count
    bias = r.normal(size=E).astype(np.float32)
    dev = torch.from_numpy(bias).cuda()
    out = torch.full((E,), float("nan"), device="cuda")
    moe.moe_bias_update(torch.from_numpy(counts).cuda(), 0.01, dev, out)
    want = ro.bias_step(bias, counts[:E], float(np.float32(0.01)))
    close(out, want, U * np.abs(want), "bias")
    moe.moe_bias_update(torch.from_numpy(counts[:E]).cuda(), 0.01, dev, dev)
    assert torch.equal(dev, out)
    big = torch.full((E,), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    big[0] -= 1 if E > 1 else 0
    moe.moe_bias_update(big, 1.0, torch.zeros(E, device="cuda"), out)
    assert out.cpu().tolist() == [1.0 if E > 1 else 0.0] + [-1.0] * (E - 1)


def test_selection_is_moe_routes_where_the_scores_say_the_same():
    """Without bias and groups, sigmoid and softmax order experts as the logits do, and a renormalised softmax has moe_route's weights."""
    for T in (17, 900):
        L, _ = _logits(T, 48, T)
        logits = torch.from_numpy(L).cuda()
        shape, a, ws = _route(logits, moe.make_scores("softmax"), None, 4, 12, 12)
        b = moe.alloc_saved(shape, keep_xp=False)
        moe.moe_route(shape, logits, b, ws)
        for n in ("topk_idx", "counts", "offsets", "row_of"):
            assert torch.equal(getattr(a, n), getattr(b, n)), n
        assert (a.topk_w - b.topk_w).abs().max() < 8 * U


@pytest.mark.parametrize("mode", [moe.MODE_SERIALIZED, moe.MODE_PERSISTENT])
@pytest.mark.parametrize("T", [20, 700])
def test_layer_behind_it(T, mode):
    """The layer on these tables is the oracle's with these weights, as separate launches and as one."""
    H, I, E, El, base, k = 128, 64, 16, 10, 3, 3
    r = np.random.default_rng(T)
    x, w1, w2 = (torch.from_numpy(r.normal(size=s).astype(np.float32)).cuda().to(torch.bfloat16) * f
                 for s, f in (((T, H), 1), ((El, H, 2 * I), H ** -0.5), ((El, I, H), I ** -0.5)))
    L, _ = _logits(T, E, T)
    bias = (0.3 * r.normal(size=E)).astype(np.float32)
    shape = moe.make_shape(T, H, I, E, El, base, k, torch.bfloat16)
    saved, ws, out = moe.alloc_saved(shape), moe.alloc_workspace(shape), torch.empty_like(x)
    scores = moe.make_scores("sigmoid", 4, 2, True, 2.0)
    moe.moe_route_scores(shape, scores, torch.from_numpy(L).cuda(), torch.from_numpy(bias).cuda(), saved, ws, mode)
    moe.moe_dispatch_to_combine(shape, x, w1, w2, out, saved, ws, mode)
    torch.cuda.synchronize()
    assert moe.moe_ffn_last_status(shape, ws) == 0
    idx, s = ro.select(L, "sigmoid", k, bias, 4, 2)
    w = ro.weights(s, idx, True, 2.0)
    want = np.zeros((T, H))
    for e in range(El):
        t, j = np.nonzero(idx == base + e)
        h = f64(x)[t] @ f64(w1)[e]
        want_e = (h[:, :I] / (1 + np.exp(-h[:, :I])) * h[:, I:]) @ f64(w2)[e]
        np.add.at(want, t, w[t, j][:, None] * want_e)
    assert np.abs(f64(out) - want).max() <= 1e-2 * np.abs(want).max()
    # with 4-bit experts: the bf16 layer on the weights that the blocks stand for
    blocks, back = [], []
    for v in (w1, w2):
        q, sc = moe.alloc_w4(*v.shape)
        moe.moe_quantize_w4(v, q, sc)
        blocks += [q, sc]
        from oracle import block_oracle as bo
        back.append(torch.from_numpy(bo.dequantize_w4(q.cpu().numpy(), sc.cpu().numpy())).cuda().to(torch.bfloat16))
    moe.moe_route_scores(shape, scores, torch.from_numpy(L).cuda(), torch.from_numpy(bias).cuda(), saved, ws)
    moe.moe_dispatch_to_combine(shape, x, back[0].contiguous(), back[1].contiguous(), out, saved, ws, moe.MODE_SERIALIZED)
    got = torch.full_like(out, float("nan"))
    moe.moe_dispatch_to_combine_w4(shape, x, *blocks, got, saved, ws)
    assert np.abs(f64(got) - f64(out)).max() <= 1e-2 * np.abs(f64(out)).max()


def test_replays_from_a_graph():
    T, E, k = 300, 64, 6
    shape = moe.make_shape(T, 64, 64, E, 16, 8, k, torch.bfloat16)
    saved, ws = moe.alloc_saved(shape, keep_xp=False), moe.alloc_workspace(shape)
    scores = moe.make_scores("sigmoid", 8, 3, True, 2.5)
    L = [torch.from_numpy(_logits(T, E, i)[0]).cuda() for i in range(3)]
    logits, bias, dw, d = L[0].clone(), torch.zeros(E, device="cuda"), torch.randn(T, k, device="cuda"), torch.empty(T, E, device="cuda")
    counts = torch.randint(0, 9, (E,), device="cuda").int()

    def step():
        moe.moe_route_scores(shape, scores, logits, bias, saved, ws)
        moe.moe_route_scores_backward(scores, logits, saved.topk_idx, dw, None, d)
        moe.moe_bias_update(counts, 0.01, bias, bias)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for i in (1, 2, 0, 1):
        logits.copy_(L[i])
        start = bias.clone()
        d.fill_(-1), saved.topk_idx.fill_(-1), saved.row_of.fill_(-9)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (d, saved.topk_idx, saved.topk_w, saved.row_of, saved.offsets, bias)]
        bias.copy_(start)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (d, saved.topk_idx, saved.topk_w, saved.row_of, saved.offsets, bias)))
