"""The 4-bit layer in every form that its products take, at widths where a wave has several steps of K: routed, rows through the permutation,
rows in tiles; 16 and 32 rows at a time; two and four column blocks per item.  Against the fp64 oracle."""
import functools

import numpy as np
import pytest
import torch

import oracle
import paper_2605_23764_amd as moe
from block_common import U, f64
from oracle import block_oracle as bo
from test_gpu_w4 import _blocks
from workloads import MoeConfig, make_inputs

pytestmark = pytest.mark.gpu

# (H, I, E, local, first, k).  A step is 128 k and four waves share them: H = 1088 has 9 steps (2, 2, 2, 3), the last of two blocks, I = 704
# 6 steps (1, 2, 1, 2), the last of two; H = 2048 16 (4 each), I = 1408 11 (2, 3, 3, 3); H = 7168 56 (14 each).
LAYERS = {
    "mid": (2048, 1408, 4, 4, 0, 2),
    "odd": (1088, 704, 12, 4, 5, 4),
    "deep": (7168, 192, 3, 2, 1, 1),
    "many": (512, 256, 64, 64, 0, 4),          # 64 experts x 8 items in both products: four column blocks
    "wide": (1088, 704, 32, 32, 0, 4),         # 32 x 22 and 32 x 17 items: four column blocks, several steps
    "few": (192, 320, 16, 2, 7, 6),            # fewer local experts than selections of a token
}


@functools.lru_cache(maxsize=2)
def _layer(name):
    """Blocks of one layer's weights on the device and what they stand for."""
    H, I, E, El, base, k = LAYERS[name]
    inp = make_inputs(MoeConfig("w4", 1, H, I, E, El, base, k, "bf16", 4000 + H + E))
    blocks, weights = [], []
    for n in ("w_gate_up", "w_down"):
        q, s = _blocks(torch.from_numpy(inp[n]).cuda())
        blocks += [q, s]
        weights.append([bo.dequantize_w4(q[e:e + 1].cpu().numpy(), s[e:e + 1].cpu().numpy())[0] for e in range(El)])
    return blocks, weights


def _bf16(a):
    return torch.from_numpy(a).to(torch.bfloat16).double().numpy()


def _expected(x, logits, weights, k, base):
    """(oracle's intermediates, the output on A as the layer rounds it, a bound of the layer's error).  GEMM-1's fp32 sums of a row have as
    many roundings as x has entries that are not zero (few here, so that the bound is sharp and a block of k left out shows), SwiGLU's
    exponential and reciprocal 4 steps of fp32 each; A is then the bf16 value, or its neighbour where a border lies within that error;
    GEMM-2's sums have I roundings, Combine some, the output one to bf16."""
    ref = oracle.forward(x, logits, *weights, k, base, len(weights[0]))
    I, off = ref["A"].shape[1], ref["offsets"]
    out, bound = np.zeros_like(ref["out"]), np.zeros_like(ref["out"])
    for e, (w1, w2) in enumerate(zip(*weights)):
        lo, hi = off[e], off[e + 1]
        if lo == hi:
            continue
        xs, g, u, a = ref["Xp"][lo:hi], ref["H1"][lo:hi, :I], ref["H1"][lo:hi, I:], ref["A"][lo:hi]
        at = np.nonzero((xs != 0).any(0))[0]
        mass = np.abs(xs[:, at]) @ np.abs(w1[at]) * ((xs != 0).sum(1, keepdims=True) * U)
        sg = 1 / (1 + np.exp(-g))
        e_a = np.abs(u) * (sg + np.abs(g) * sg * (1 - sg)) * mass[:, :I] + np.abs(g * sg) * mass[:, I:] + 8 * U * (1 + np.abs(g)) * np.abs(a)
        ab = _bf16(a)
        e_a = np.maximum(_bf16(a + e_a) - ab, ab - _bf16(a - e_a))
        t, j = ref["token_of"][lo:hi], ref["slot_of"][lo:hi]
        w = ref["topk_w"][t, j][:, None]
        out[t] += w * (ab @ w2)                                          # a token is in an expert's rows once
        bound[t] += w * ((e_a + (I + 8) * U * (np.abs(ab) + e_a)) @ np.abs(w2))
    return ref, out, bound + 2.0 ** -8 * (np.abs(out) + bound)


def _tokens(T, H, E, seed):
    """x with an entry in 16 that is not zero, logits; on the device and as the oracle takes them."""
    g = torch.Generator("cuda").manual_seed(seed)
    x = 4 * torch.randn(T, H, generator=g, device="cuda") * (torch.rand(T, H, generator=g, device="cuda") < 1 / 16)
    x, logits = x.to(torch.bfloat16), torch.randn(T, E, generator=g, device="cuda")
    return x, logits


def _call(shape, x, logits, blocks, saved):
    ws = moe.alloc_workspace(shape)
    ws.fill_(255)                                  # not a number, should anything be read that was not written
    out = torch.full((shape.T, shape.H), float("nan"), dtype=torch.bfloat16, device="cuda")
    moe.moe_ffn_forward_w4(shape, x, logits, *blocks, out, saved, ws)
    torch.cuda.synchronize()
    assert moe.moe_ffn_last_status(shape, ws) == 0
    return out


# rows of an expert on average T k / E: up to 8 sixteen at a time, above 16 in tiles; up to 16 tokens (of up to 64 experts) routed
@pytest.mark.parametrize("name,T", [
    ("mid", 1), ("mid", 5), ("mid", 16),           # routed
    ("mid", 17), ("mid", 24), ("mid", 32),         # through the permutation: rows 8 (16 at a time), 12 and 16 (32 at a time)
    ("mid", 40), ("mid", 133),                     # tiles: rows 20 and 66
    ("odd", 1), ("odd", 16), ("odd", 25), ("odd", 40), ("odd", 60), ("odd", 200),
    ("deep", 2), ("deep", 16), ("deep", 26), ("deep", 29), ("deep", 70),
    ("many", 1), ("many", 16), ("many", 30), ("many", 128), ("many", 150), ("many", 300),
    ("wide", 2), ("wide", 16), ("wide", 40), ("wide", 100), ("wide", 150),
    ("few", 1), ("few", 16), ("few", 20), ("few", 40), ("few", 200)])
def test_forms(name, T):
    H, I, E, El, base, k = LAYERS[name]
    print(f"4-bit layer {name} T={T}", flush=True)
    blocks, weights = _layer(name)
    x, logits = _tokens(T, H, E, 31 * T + H)
    shape = moe.make_shape(T, H, I, E, El, base, k, torch.bfloat16)
    ref, want, tol = _expected(f64(x), f64(logits), weights, k, base)
    out = _call(shape, x, logits, blocks, None)
    err = np.abs(f64(out) - want)
    assert (err <= tol).all(), np.nanmax(err / np.maximum(tol, 1e-300))
    saved = moe.alloc_saved(shape)
    again = _call(shape, x, logits, blocks, saved)                     # with a routing launch: the same sums in the same order
    assert torch.equal(again, out)
    np.testing.assert_array_equal(saved.row_of.cpu().numpy(), ref["row_of"])
    assert torch.equal(_call(shape, x, logits, blocks, None), out)


@pytest.mark.parametrize("T", [16, 100, 128])
def test_one_busy_expert(T):
    """All tokens to one expert beside many idle ones: more rows than the average promises, in the forms of few rows."""
    H, I, E, El, base, _ = LAYERS["many"]
    blocks, weights = _layer("many")
    x, logits = _tokens(T, H, E, T)
    logits[:, 9] += 50.0
    out = _call(moe.make_shape(T, H, I, E, El, base, 1, torch.bfloat16), x, logits, blocks, None)
    ref, want, tol = _expected(f64(x), f64(logits), weights, 1, base)
    assert ref["counts"][9] == T and (np.abs(f64(out) - want) <= tol).all()


@pytest.mark.parametrize("T", [4095, 4096])
def test_tokens_of_two_gigabytes(T):
    """x at and just below 2^31 bytes: through the permutation with 31-bit offsets below, in tiles from there on."""
    H, I, E, base = 262144, 64, 256, 37
    print(f"4-bit layer T={T} H={H}", flush=True)
    g = torch.Generator("cuda").manual_seed(T)
    x = torch.zeros(T, H, dtype=torch.bfloat16, device="cuda")
    for i in range(0, T, 512):
        n = min(512, T - i)
        x[i:i + n] = 32 * torch.randn(n, H, generator=g, device="cuda") * (torch.rand(n, H, generator=g, device="cuda") < 1 / 1024)
    logits = torch.randn(T, E, generator=g, device="cuda")
    logits[:, base] -= 100.0
    mine = torch.tensor([0, 1, 63, 1000, 2047, 2048, T - 2, T - 1], device="cuda")
    logits[mine, base] = 100.0
    blocks = [b for K, N in ((H, 2 * I), (I, H)) for b in _blocks(torch.randn(1, K, N, generator=g, device="cuda") * K ** -0.5)]
    weights = [[bo.dequantize_w4(q.cpu().numpy(), s.cpu().numpy())[0]] for q, s in (blocks[:2], blocks[2:])]
    out = _call(moe.make_shape(T, H, I, E, 1, base, 1, torch.bfloat16), x, logits, blocks, None)
    _, want, tol = _expected(f64(x[mine]), f64(logits[mine]), weights, 1, base)
    assert (np.abs(f64(out[mine]) - want) <= tol).all()
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[mine] = False
    assert all((out[i:i + 512][rest[i:i + 512]] == 0).all() for i in range(0, T, 512))
