"""The gradient of the routing by scores at its edges: selected scores whose sum is subnormal in 64 bits, gradients of slots that have no part, an
expert that two slots of a token name."""
import numpy as np
import pytest
import torch

import paper_2605_23764_amd as moe
from block_common import U, f64
from oracle import router_oracle as ro

pytestmark = pytest.mark.gpu


def _gradient(scores, L, idx, dw, dadd=None):
    dev = [None if a is None else torch.from_numpy(np.ascontiguousarray(a, dtype=t)).cuda()
           for a, t in ((L, np.float32), (idx, np.int32), (dw, np.float32), (dadd, np.float32))]
    got = torch.full(L.shape, float("nan"), device="cuda")
    moe.moe_route_scores_backward(scores, *dev, got)
    return f64(got)


@pytest.mark.parametrize("E,k", [(8, 3), (24, 6), (64, 8), (100, 5), (256, 16)])
@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
def test_sums_that_are_subnormal(kind, E, k):
    """Renormalised scores below 2^-1022.  Far below zero a sigmoid is exp(l), and a softmax is exp(l - the row's largest), which a bias keeps out of
    the selection: the weights are those of a softmax over the selected alone.

    Tolerance: a subnormal score is a multiple of 2^-1074, so the kernel's and numpy's are one such step apart at most, beside 4 roundings of
    2^-53 each of ordinary arithmetic; w = s / sum is off by that of its own score and of the sum's.  dl = scale w (dw - sum w dw) then is off by
    w (r_w |dw - d| + sum of r_w w |dw|), and rounded once to 32 bits."""
    T = 70
    r = np.random.default_rng(E + k)
    L = r.uniform(-736, -712, size=(T, E)).astype(np.float32)
    if kind == "softmax":
        L[:, 0] = 0.0                                               # the largest: what the selection leaves out
    idx = np.stack([1 + r.permutation(E - 1)[:k] for _ in range(T)])
    dw = r.normal(size=(T, k)).astype(np.float32)
    got = _gradient(moe.make_scores(kind, renormalize=True, scale=1.5), L, idx, dw)
    assert np.isfinite(got).all()
    s = np.exp(np.take_along_axis(L.astype(np.float64), idx, 1))
    total = s.sum(1, keepdims=True)
    assert (total < 2.0 ** -1022).all() and (total > 0).all()
    w = s / total
    step = 2.0 ** -1074
    r_w = step / s + (k * step) / total + 8 * 2.0 ** -53
    d = (w * dw).sum(1, keepdims=True)
    e_d = (r_w * w * np.abs(dw)).sum(1, keepdims=True)
    want, tol = np.zeros((T, E)), np.zeros((T, E))
    np.put_along_axis(want, idx, 1.5 * w * (dw - d), 1)
    np.put_along_axis(tol, idx, 1.5 * w * (r_w * np.abs(dw - d) + e_d), 1)
    # a softmax's other experts: what the sum over the selected takes off them is 0
    assert (np.abs(got - want) <= tol * 1.01 + U * np.abs(want) + 2.0 ** -149).all(), np.abs(got - want).max()
    # the forward on the same logits gives these weights
    bias = np.full(E, -3.0, dtype=np.float32)
    bias[idx[0]] = np.linspace(2.0, 1.0, k).astype(np.float32)
    shape = moe.make_shape(1, 64, 64, E, E, 0, k, torch.bfloat16)
    saved, ws = moe.alloc_saved(shape, keep_xp=False), moe.alloc_workspace(shape)
    moe.moe_route_scores(shape, moe.make_scores(kind, renormalize=True, scale=1.5), torch.from_numpy(L[:1]).cuda(), torch.from_numpy(bias).cuda(), saved, ws)
    np.testing.assert_array_equal(saved.topk_idx.cpu().numpy()[0], idx[0])
    assert (np.abs(f64(saved.topk_w)[0] - 1.5 * w[0]) <= 1.5 * w[0] * (r_w[0] * 1.01 + U)).all()


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renorm", [True, False], ids=["renorm", "plain"])
@pytest.mark.parametrize("T,E,k", [(70, 24, 4), (33, 256, 8), (5, 3, 2)])
def test_slots_without_a_part_may_hold_anything(T, E, k, kind, renorm):
    """Ids outside 0 .. E - 1, and experts whose logit is -inf: whatever their gradient holds, the others' are those of the slots that count."""
    r = np.random.default_rng(T)
    L = r.normal(size=(T, E)).astype(np.float32)
    idx, _ = ro.select(L, kind, k)
    dw = r.normal(size=(T, k)).astype(np.float32)
    clean = dw.copy()
    bad = [float("nan"), float("inf"), -float("inf"), 3e38]
    for i, t in enumerate(range(0, T, 2)):
        j = i % k
        if i % 3 == 2:
            L[t, idx[t, j]] = -np.inf if i % 2 else np.nan
        else:
            idx[t, j] = (-1, E, -7, 2 ** 31 - 1)[i % 4]
        dw[t, j], clean[t, j] = bad[i % 4], 0.0
    scores = moe.make_scores(kind, renormalize=renorm, scale=1.25)
    got = _gradient(scores, L, idx, dw)
    np.testing.assert_array_equal(got, _gradient(scores, L, idx, clean))
    want = ro.weights_backward(L.astype(np.float64), kind, idx, clean.astype(np.float64), renorm, 1.25)
    assert np.abs(got - want).max() <= 40 * U * np.abs(clean).max() * 1.25


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renorm", [True, False], ids=["renorm", "plain"])
@pytest.mark.parametrize("E,k", [(3, 3), (8, 8), (24, 5), (64, 6), (256, 16)])
def test_an_expert_named_twice(E, k, kind, renorm):
    """Its slots' parts add up."""
    T = 50
    r = np.random.default_rng(E)
    L = r.normal(size=(T, E)).astype(np.float32)
    idx = r.integers(0, E, size=(T, k))
    idx[:, 1] = idx[:, 0]
    idx[::3] = idx[::3, :1]                                         # all the same
    dw, dadd = (r.normal(size=s).astype(np.float32) for s in ((T, k), (T, E)))
    scores = moe.make_scores(kind, renormalize=renorm, scale=1.25)
    want = ro.weights_backward(L.astype(np.float64), kind, idx, dw.astype(np.float64), renorm, 1.25)
    tol = 40 * U * np.abs(dw).max() * 1.25
    assert np.abs(_gradient(scores, L, idx, dw) - want).max() <= tol * (1 + k)         # k parts, each rounded, and their sums
    assert np.abs(_gradient(scores, L, idx, dw, dadd) - (want + dadd)).max() <= tol * (1 + k) + U * np.abs(dadd).max() * 2
