"""4-bit experts on the GPU: the quantiser against the oracle, code for code; the layer against the fp64 oracle on the weights that the blocks
stand for, from one token to more rows per expert than are in hand at a time."""
import numpy as np
import pytest
import torch

import oracle
import paper_2605_23764_amd as moe
from block_common import U, f64
from oracle import block_oracle as bo
from workloads import MoeConfig, make_inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("E,K,N", [(1, 32, 1), (3, 64, 40), (2, 1088, 33), (5, 96, 257)])
def test_quantize(E, K, N, dtype):
    r = np.random.default_rng(K + N)
    w = r.normal(size=(E, K, N)) * np.exp(3 * r.normal(size=(E, 1, N)))
    w[0, :32, 0] = 0.0
    if N > 1:
        w[:, 3::7, 1] = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0])[np.arange(len(range(3, K, 7))) % 8]   # ties
        w[:, 0::32, 1] = 4.0
    if N > 30:
        w[0, 5, 2], w[0, 40 % K, 3], w[0, 9, 4] = np.inf, np.nan, -np.inf
        w[0, :, 5], w[0, :, 6], w[0, :, 7] = 1e-38 * w[0, :, 5], 3e38, 1e-44
    t = torch.from_numpy(w.astype(np.float32)).cuda().to(dtype)
    q, s = moe.alloc_w4(E, K, N)
    q.fill_(99), s.fill_(99)
    moe.moe_quantize_w4(t, q, s)
    wq, ws = bo.quantize_w4(f64(t))
    np.testing.assert_array_equal(s.cpu().numpy(), ws)
    np.testing.assert_array_equal(q.cpu().numpy()[ws != 255], wq[ws != 255])


def _blocks(w):
    q, s = moe.alloc_w4(*w.shape)
    moe.moe_quantize_w4(w, q, s)
    return q, s


def _run(cfg, dev, saved=None):
    shape = moe.make_shape(cfg.T, cfg.H, cfg.I, cfg.E, cfg.E_local, cfg.expert_base, cfg.k, torch.bfloat16)
    ws = moe.alloc_workspace(shape)
    ws.fill_(255)                                  # not a number, should anything be read that was not written
    out = torch.full((cfg.T, cfg.H), float("nan"), dtype=torch.bfloat16, device="cuda")
    moe.moe_ffn_forward_w4(shape, dev["x"], dev["logits"], *dev["w1"], *dev["w2"], out, saved, ws)
    torch.cuda.synchronize()
    return shape, out


def _device(inp):
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    return dict(x=up(inp["x"]).to(torch.bfloat16), logits=up(inp["logits"]), w1=_blocks(up(inp["w_gate_up"])), w2=_blocks(up(inp["w_down"])))


def _bound(ref, w1, w2, cfg):
    """Of |out - oracle|: GEMM-1's and GEMM-2's fp32 sums over K terms, A's rounding to bf16 (half a step, carried through the weights of
    GEMM-2), SwiGLU's exponential and reciprocal (4 steps of fp32), Combine's k terms, the output's rounding."""
    bound = np.zeros_like(ref["out"])
    off = ref["offsets"]
    for e in range(cfg.E_local):
        for r in range(off[e], off[e + 1]):
            x, t, j = ref["Xp"][r], ref["token_of"][r], ref["slot_of"][r]
            g, u = ref["H1"][r][:cfg.I], ref["H1"][r][cfg.I:]
            mass = np.abs(x) @ np.abs(w1[e]) * (cfg.H * U)
            sg = 1 / (1 + np.exp(-g))
            e_a = np.abs(u) * (sg + np.abs(g) * sg * (1 - sg)) * mass[:cfg.I] + np.abs(g * sg) * mass[cfg.I:] + 8 * U * (1 + np.abs(g)) * np.abs(g * sg * u)
            e_a = e_a + 2.0 ** -8 * (np.abs(ref["A"][r]) + e_a)
            bound[t] += ref["topk_w"][t, j] * (e_a @ np.abs(w2[e]) + (cfg.I + 8) * U * (np.abs(ref["A"][r]) @ np.abs(w2[e])))
    return bound + 2.0 ** -8 * (np.abs(ref["out"]) + bound)


@pytest.mark.parametrize("T,H,I,E,El,base,k", [
    (1, 64, 64, 4, 4, 0, 1), (1, 192, 64, 8, 3, 2, 2), (2, 320, 192, 8, 8, 0, 2), (7, 128, 448, 16, 5, 11, 3), (16, 256, 128, 4, 4, 0, 4),
    (33, 64, 256, 4, 2, 1, 2), (64, 448, 64, 6, 6, 0, 3), (65, 192, 192, 8, 8, 0, 8), (150, 128, 128, 4, 4, 0, 2), (300, 64, 64, 3, 1, 1, 1)])
def test_layer(T, H, I, E, El, base, k):
    print(f"4-bit layer T={T} H={H} I={I} E={E} local {El} from {base} k={k}", flush=True)
    cfg = MoeConfig("w4", T, H, I, E, El, base, k, "bf16", 900 + T)
    inp = make_inputs(cfg)
    dev = _device(inp)
    w1, w2 = (bo.dequantize_w4(q.cpu().numpy(), s.cpu().numpy()) for q, s in (dev["w1"], dev["w2"]))
    ref = oracle.forward(inp["x"], inp["logits"], w1, w2, cfg.k, cfg.expert_base, cfg.E_local)
    shape, out = _run(cfg, dev)
    err, tol = np.abs(f64(out) - ref["out"]), _bound(ref, w1, w2, cfg)
    assert (err <= tol).all(), np.nanmax(err / np.maximum(tol, 1e-300))
    saved = moe.alloc_saved(shape)
    _, again = _run(cfg, dev, saved)
    assert torch.equal(again, out)
    np.testing.assert_array_equal(saved.row_of.cpu().numpy(), ref["row_of"])
    np.testing.assert_array_equal(saved.topk_idx.cpu().numpy(), ref["topk_idx"])


def test_every_code_and_scale():
    """One-hot tokens, gate 96 (whose sigmoid is 1), W_down the identity: out = 96 * code * 2^(s - 127), exact, for every scale that keeps
    that finite; beyond, infinities; scale 255 is not a number."""
    H = I = 64
    x = torch.eye(H, dtype=torch.bfloat16, device="cuda")
    shape = moe.make_shape(H, H, I, 1, 1, 0, 1, torch.bfloat16)
    ws = moe.alloc_workspace(shape)
    logits = torch.zeros(H, 1, device="cuda")
    code = (torch.arange(I)[None, :] + torch.arange(H)[:, None]) % 16                       # [k, n]
    c = code.view(2, 32, I).permute(0, 2, 1)
    q1 = torch.full((1, 2, 2 * I, 16), 0x77, dtype=torch.uint8)
    q1[0, :, I:] = (c[..., 0::2] | c[..., 1::2] << 4).to(torch.uint8)
    s1 = torch.full((1, 2, 2 * I), 131, dtype=torch.uint8)
    w2 = torch.eye(I, device="cuda")[None]
    q2, s2 = _blocks(w2)
    values = np.concatenate([bo.E2M1, -bo.E2M1])[code.numpy()]
    for s in [*range(0, 246), 255]:
        s1[0, :, I:] = s
        out = torch.empty(H, H, dtype=torch.bfloat16, device="cuda")
        moe.moe_ffn_forward_w4(shape, x, logits, q1.cuda(), s1.cuda(), q2, s2, out, None, ws)
        if s == 255:
            assert torch.isnan(out.float()).all()
        else:
            np.testing.assert_array_equal(f64(out), 96.0 * values * 2.0 ** (s - 127), err_msg=str(s))


@pytest.mark.parametrize("T,E,El,base,k", [(1, 256, 32, 0, 8), (4, 250, 100, 150, 16), (5, 130, 130, 0, 3), (16, 64, 64, 0, 2), (16, 5, 5, 0, 1),
                                           (8, 100, 60, 17, 9), (17, 64, 20, 3, 4)])
def test_few_tokens_route_alike(T, E, El, base, k):
    """Few tokens take no routing launch unless a MoeSaved asks for its results: the same bits both ways, ties, zeros of both signs,
    infinities and NaN among the logits included."""
    cfg = MoeConfig("w4", T, 128, 64, E, El, base, k, "bf16", 70 + T)
    inp = make_inputs(cfg)
    r = np.random.default_rng(E)
    lg = np.round(inp["logits"] * 2) / 2                             # many ties
    lg[r.random(lg.shape) < 0.1] = -0.0
    if k < E // 2:
        lg[r.random(lg.shape) < 0.05] = -np.inf
        lg[r.random(lg.shape) < 0.05] = np.nan
    inp["logits"] = lg
    dev = _device(inp)
    shape, out = _run(cfg, dev)
    _, want = _run(cfg, dev, moe.alloc_saved(shape))
    assert torch.equal(out, want) and not torch.isnan(out.float()).any()


def test_tokens_without_a_local_expert():
    cfg = MoeConfig("w4", 40, 64, 64, 16, 2, 14, 1, "bf16", 3)
    inp = make_inputs(cfg)
    inp["logits"][:, 14:] -= 100.0
    _, out = _run(cfg, _device(inp))
    assert (out == 0).all()


def test_weights_of_an_idle_expert_are_not_used():
    """An expert without rows may hold anything."""
    cfg = MoeConfig("w4", 6, 128, 64, 4, 4, 0, 2, "bf16", 4)
    inp = make_inputs(cfg)
    inp["logits"][:, 2] = -50.0
    dev = _device(inp)
    _, want = _run(cfg, dev)
    for q, s in (dev["w1"], dev["w2"]):
        s[2] = 255
    _, out = _run(cfg, dev)
    assert torch.equal(out, want) and not torch.isnan(out.float()).any()


def test_replays_from_a_graph():
    cfg = MoeConfig("w4", 20, 256, 128, 8, 8, 0, 2, "bf16", 5)
    dev = _device(make_inputs(cfg))
    shape = moe.make_shape(cfg.T, cfg.H, cfg.I, cfg.E, cfg.E_local, cfg.expert_base, cfg.k, torch.bfloat16)
    ws, out = moe.alloc_workspace(shape), torch.empty(cfg.T, cfg.H, dtype=torch.bfloat16, device="cuda")

    def step():
        moe.moe_ffn_forward_w4(shape, dev["x"], dev["logits"], *dev["w1"], *dev["w2"], out, None, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for seed in (1, 2, 1):
        g = torch.Generator("cuda").manual_seed(seed)
        dev["x"].copy_(torch.randn(cfg.T, cfg.H, generator=g, device="cuda"))
        dev["logits"].copy_(torch.randn(cfg.T, cfg.E, generator=g, device="cuda"))
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and not torch.isnan(got.float()).any()
