"""The operators together: a pre-norm MoE block's training step and its decode step, against the oracles put together in fp64."""
import numpy as np
import pytest
import torch

import oracle
from block_common import f64
from gpu_common import TOL, rel_err
from oracle import block_oracle as bo
from paper_2605_23764_amd.moe_block import MoeBlock

pytestmark = pytest.mark.gpu


def _expected(b, x, dout, dz, mask):
    """Forward and backward on the logits that the block has computed (so that the selections are the same)."""
    seed, offset = (int(v) for v in b.rng.tolist())
    p64 = {n: f64(getattr(b, n)) for n in ("w_router", "w_gate_up", "w_down", "gamma", "beta", "gamma_next", "beta_next", "logits")}
    y, mean, rstd = bo.layer_norm(x, p64["gamma"], p64["beta"], b.eps)
    f = oracle.forward(y, p64["logits"], p64["w_gate_up"], p64["w_down"], b.k, 0, b.E)
    keep = bo.dropout_factor(b.T, b.H, b.p, seed, offset)
    z = x + f["out"] * keep
    out, mean2, rstd2 = bo.layer_norm(z, p64["gamma_next"], p64["beta_next"], b.eps)
    counts, n, _, loss = bo.balance(p64["logits"], f["topk_idx"], mask, b.coef)
    gz, dgn, dbn = bo.layer_norm_backward(dout, z, p64["gamma_next"], mean2, rstd2, dz)
    g = oracle.backward(gz * keep, f, p64["w_gate_up"], p64["w_down"])
    dl = bo.router_backward(p64["logits"], f["topk_idx"], f["topk_w"], g["d_topk_w"], mask, b.coef, counts, n)
    dx, dg, db = bo.layer_norm_backward(g["dX"] + dl @ p64["w_router"].T, x, p64["gamma"], mean, rstd, gz)
    return dict(z=z, out=out, loss=np.array([loss]), dx=dx, dz=gz, dm=gz * keep, dgamma=dg, dbeta=db, dgamma_next=dgn, dbeta_next=dbn,
                dlogits=dl, dw_router=y.T @ dl, dw_gate_up=g["dW_gate_up"], dw_down=g["dW_down"]), counts


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,H,I,E,k,masked", [(96, 128, 64, 8, 2, False), (333, 192, 128, 12, 3, True)])
def test_training_step(T, H, I, E, k, masked, dtype):
    print(f"block T={T} H={H} I={I} E={E} k={k} {dtype}", flush=True)
    r = np.random.default_rng(T)
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    b = MoeBlock(T, H, I, E, k, dtype=tdt, p=0.2, coef=0.3, seed=5)
    b.gamma.copy_(torch.from_numpy(1 + 0.2 * r.normal(size=H)))
    b.beta_next.copy_(torch.from_numpy(0.3 * r.normal(size=H)))
    x, dout, dz = (torch.from_numpy(r.normal(size=(T, H)).astype(np.float32)).cuda().to(tdt) for _ in range(3))
    mask = torch.from_numpy((r.random(T) < 0.7)).cuda() if masked else None
    for step in range(2):
        b.step(x, dout, dz, mask)
        want, counts = _expected(b, f64(x), f64(dout), f64(dz), None if mask is None else mask.cpu().numpy())
        assert b.counts[:-1].cpu().tolist() == counts.tolist()
        # norm, layer and norm follow each other: the layer's tolerance three times, twice that where the whole backward lies behind
        for name, ref in want.items():
            tol = TOL[dtype] * (3 if name in ("z", "out", "loss", "dz", "dm", "dgamma_next", "dbeta_next") else 6)
            err = rel_err(f64(getattr(b, name)), ref)
            assert err <= tol, f"step {step}, {name}: {err:.2e} > {tol}"


def test_decode_step():
    """On the weights that the blocks stand for; tokens one and several at a time give the same rows."""
    b = MoeBlock(64, 256, 128, 8, 2, seed=9)
    b.quantize()
    x = torch.randn(33, 256, generator=torch.Generator("cuda").manual_seed(2), device="cuda").to(torch.bfloat16)
    z = b.decode(x)
    w1, w2 = (bo.dequantize_w4(q.cpu().numpy(), s.cpu().numpy()) for q, s in (b.blocks[:2], b.blocks[2:]))
    y = bo.layer_norm(f64(x), f64(b.gamma), f64(b.beta), b.eps)[0]
    yb = f64(torch.from_numpy(y).to(torch.bfloat16))
    logits = yb @ f64(b.w_router)
    order = np.sort(logits, axis=1)
    clear = order[:, -b.k] - order[:, -b.k - 1] > 0.05                 # the selection does not hang on a rounding of y
    assert clear.sum() > 20
    want = f64(x) + oracle.forward(yb, logits, w1, w2, b.k, 0, b.E)["out"]
    assert rel_err(f64(z)[clear], want[clear]) <= 3 * TOL["bf16"]
    assert torch.equal(b.decode(x[:1]), z[:1])
