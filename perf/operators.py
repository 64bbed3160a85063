"""Timed cases of the operators around the MoE-FFN layer in a transformer block, in plain torch and through the public entry points.

What a program does with them, and the case kind that stands for it:
  norm            layer norm in front of the layer, inference (one call)
  norm_train      its forward and backward; the gradient that came along the residual path joins in the backward
  drop            dropout of the layer's output + residual, forward and backward
  drop_norm       the same with the next block's layer norm in one call, forward and backward
  balance         balance loss and per-expert counts of a batch, no gradients (monitoring while serving or evaluating)
  balance_train   the same with the gradient of the logits: that of the loss plus that of the routing weights
  w4              a serving step of the layer with 4-bit expert weights
"""
from __future__ import annotations

import math

import torch

own = False      # True: run() calls the framework's operators

# One GPU's share of a layer: hidden size, expert width, experts, local experts, first local expert, experts per token.
MID = dict(H=2048, I=1408, E=16, E_local=16, base=0, k=4)         # mid-size layer, every expert local
LARGE = dict(H=7168, I=2048, E=256, E_local=32, base=0, k=8)      # 256 experts over eight GPUs
ODD = dict(H=1088, I=704, E=24, E_local=10, base=6, k=3)          # width not a multiple of a tile, experts from the middle

EPS = 1e-5
COEF = 0.01


def _rows(name, kind, T, H, dtype="bf16", p=0.0):
    return dict(name=name, kind=kind, T=T, H=H, dtype=dtype, p=p)


def _router(name, kind, T, E, k, masked=0.0):
    return dict(name=name, kind=kind, T=T, E=E, k=k, masked=masked)


def _w4(name, T, layer):
    return dict(name=name, kind="w4", T=T, **layer)


def listed():
    return [
        # one token of one sequence in front of the layer: the smallest call there is
        _rows("norm_1_large", "norm", 1, 7168),
        # a training step's norm at the headline shape
        _rows("norm_train_8192_large", "norm_train", 8192, 7168),
        # fp32 storage, rows that no vector divides
        _rows("norm_train_1500_odd_f32", "norm_train", 1500, 1001, "f32"),
        # the end of a mid-size layer in training
        _rows("drop_4096_mid", "drop", 4096, 2048, p=0.1),
        # the end of one block and the start of the next at the headline shape: the largest case of these
        _rows("drop_norm_8192_large", "drop_norm", 8192, 7168, p=0.1),
        # a short fp32 batch of ordinary width
        _rows("drop_norm_600_f32", "drop_norm", 600, 1408, "f32", p=0.25),
        # router statistics of a serving batch
        _router("balance_32_large", "balance", 32, 256, 8),
        # a training step's router at the headline shape
        _router("balance_train_8192_large", "balance_train", 8192, 256, 8),
        # many tokens of padded sequences, few experts, odd count
        _router("balance_train_30001_masked", "balance_train", 30001, 64, 6, masked=0.2),
        # one token through a mid-size layer of 4-bit experts
        _w4("w4_1_mid", 1, MID),
        # a serving batch; about 20 of the 32 local experts get one or two rows each
        _w4("w4_32_large", 32, LARGE),
        # a larger batch of odd sizes; ten experts of about 12 rows
        _w4("w4_100_odd", 100, ODD),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm_train", "norm_train", "drop", "drop_norm", "drop_norm", "balance", "balance_train",
                       "balance_train", "w4", "w4", "w4"])
    if kind in ("norm", "norm_train", "drop", "drop_norm"):
        dtype = "f32" if rng.random() < 0.35 else "bf16"
        H = 64 * _log_int(rng, 1, 112) if rng.random() < 0.7 else _log_int(rng, 33, 7168)
        T = _log_int(rng, 1, 8192) if kind == "norm" else _log_int(rng, 16, 8192 if dtype == "bf16" else 4096)
        return dict(kind=kind, T=T, H=H, dtype=dtype, p=0.0 if kind.startswith("norm") else rng.choice([0.0, 0.05, 0.1, 0.3, 0.5]))
    if kind in ("balance", "balance_train"):
        E = rng.choice([8, 16, 24, 60, 64, 128, 160, 256])
        return dict(kind=kind, T=_log_int(rng, 1 if kind == "balance" else 32, 32768), E=E, k=rng.randint(1, 8),
                    masked=rng.choice([0.0, 0.0, 0.1, 0.5]))
    E = rng.choice([8, 16, 24, 64, 128])
    E_local = rng.choice([e for e in (4, 8, 10, 16, 32) if e <= E])
    layer = rng.choice([MID, LARGE, dict(H=64 * _log_int(rng, 4, 64), I=64 * _log_int(rng, 2, 32), E=E, E_local=E_local,
                                         base=rng.randint(0, E - E_local), k=rng.randint(1, 8))])
    return dict(kind=kind, T=_log_int(rng, 1, 128), **layer)


# ---- inputs ----
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _hidden(T, H, dt, g):
    """A residual stream: an offset per token, and one channel in 97 that is eight times as large as the others."""
    x = torch.randn(T, H, generator=g, device="cuda")
    x[:, 5::97] *= 8.0
    return (x + 0.3 * torch.randn(T, 1, generator=g, device="cuda")).to(dt)


def _pack_e2m1(w):
    """w [K, N] float -> (codes [K/32, N, 16] uint8, scales [K/32, N] uint8): per group of 32 k of a column the power of two that
    brings the largest magnitude into [4, 8), values rounded to {0, .5, 1, 1.5, 2, 3, 4, 6}; low nibble = even k."""
    K, N = w.shape
    v = w.view(K // 32, 32, N)
    e = torch.floor(torch.log2(v.abs().amax(1).clamp_min(2.0 ** -100))) - 2.0
    v = v / torch.exp2(e)[:, None, :]
    mid = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=w.device)
    code = torch.bucketize(v.abs(), mid) + 8 * (v < 0)
    code = code.to(torch.uint8).permute(0, 2, 1)
    return (code[..., 0::2] | (code[..., 1::2] << 4)).contiguous(), (e + 127.0).to(torch.uint8)


def prepare(case, seed):
    g = _generator(seed)
    T, kind = case["T"], case["kind"]
    s = dict(case=case)
    if kind in ("norm", "norm_train", "drop", "drop_norm"):
        H, dt = case["H"], _dtype(case)
        if kind != "drop":
            s["gamma"] = (1.0 + 0.2 * torch.randn(H, generator=g, device="cuda")).to(dt)
            s["beta"] = (0.1 * torch.randn(H, generator=g, device="cuda")).to(dt)
        s["x"] = _hidden(T, H, dt, g)                            # norm: its input; else the residual
        if kind in ("drop", "drop_norm"):
            s["v"] = torch.randn(T, H, generator=g, device="cuda").to(dt)
            s["rng"] = torch.tensor([int(seed) * 7919 + 17, 123456789012 + int(seed)], dtype=torch.int64, device="cuda")
        if kind != "norm":
            s["dy"] = torch.randn(T, H, generator=g, device="cuda").to(dt)
        if kind in ("norm_train", "drop_norm"):
            s["dres"] = (0.5 * torch.randn(T, H, generator=g, device="cuda")).to(dt)
        return s
    E, k = case["E"], case["k"]
    s["logits"] = torch.randn(T, E, generator=g, device="cuda")
    if kind in ("balance", "balance_train"):
        s["logits"] += torch.randn(E, generator=g, device="cuda")                # experts that are liked more than others
        top = torch.sort(s["logits"], dim=1, descending=True, stable=True)
        s["topk_idx"] = top.indices[:, :k].to(torch.int32).contiguous()
        s["topk_w"] = torch.softmax(top.values[:, :k], dim=1)
        s["dtopk_w"] = torch.randn(T, k, generator=g, device="cuda") / T
        s["mask"] = (torch.rand(T, generator=g, device="cuda") >= case["masked"]).to(torch.uint8) if case["masked"] else None
        s["dloss"] = torch.ones(1, device="cuda")
        return s
    H, I, El = case["H"], case["I"], case["E_local"]
    s["x"] = torch.randn(T, H, generator=g, device="cuda").to(torch.bfloat16)
    for name, K, N in (("gate_up", H, 2 * I), ("down", I, H)):
        q = torch.empty(El, K // 32, N, 16, dtype=torch.uint8, device="cuda")
        sc = torch.empty(El, K // 32, N, dtype=torch.uint8, device="cuda")
        for e in range(El):
            q[e], sc[e] = _pack_e2m1(torch.randn(K, N, generator=g, device="cuda") * K ** -0.5)
        s["q_" + name], s["s_" + name] = q, sc
    return s


# ---- the plain form ----
def _mulhilo(a, m):
    """High and low 32 bits of a * m, both below 2^32, held in int64 (the product wraps modulo 2^64)."""
    p = a * m
    return (p >> 32) & 0xFFFFFFFF, p & 0xFFFFFFFF


def _kept(s):
    """The dropout mask [T, H]: Philox4x32-10 (Salmon et al., 2011) of the counter (h / 8, t, offset), keyed by the seed."""
    T, H, p = (s["case"][n] for n in ("T", "H", "p"))
    n8 = (H + 7) // 8
    seed, off = s["rng"][0], s["rng"][1]
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    i64 = dict(dtype=torch.int64, device="cuda")
    c0 = torch.arange(n8, **i64).expand(T, n8)
    c1 = torch.arange(T, **i64)[:, None].expand(T, n8)
    c2, c3 = (off & 0xFFFFFFFF).expand(T, n8), ((off >> 32) & 0xFFFFFFFF).expand(T, n8)
    for _ in range(10):
        h0, l0 = _mulhilo(c0, 0xD2511F53)
        h1, l1 = _mulhilo(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack([c0, c1, c2, c3], dim=-1)
    u16 = torch.stack([words & 0xFFFF, words >> 16], dim=-1).view(T, n8 * 8)[:, :H]
    return u16 >= round(p * 65536)


def _drop_scale(p):
    return 65536.0 / (65536 - round(p * 65536))


def _dropped(s, v):
    return torch.where(_kept(s), v * _drop_scale(s["case"]["p"]), torch.zeros((), device="cuda")) if s["case"]["p"] > 0 else v


def _norm(x, gamma, beta):
    x = x.float()
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((d * d).mean(1) + EPS)
    return d * rstd[:, None] * gamma.float() + beta.float(), mean, rstd


def _norm_grads(dy, x, gamma, mean, rstd, dres):
    dy, xh = dy.float(), (x.float() - mean[:, None]) * rstd[:, None]
    dxh = dy * gamma.float()
    dx = rstd[:, None] * (dxh - dxh.mean(1, keepdim=True) - xh * (dxh * xh).mean(1, keepdim=True)) + dres.float()
    return dx, (dy * xh).sum(0), dy.sum(0)


def _plain_rows(s):
    kind, dt = s["case"]["kind"], s["x"].dtype
    if kind == "norm":
        y, _, _ = _norm(s["x"], s["gamma"], s["beta"])
        return dict(y=y.to(dt))
    if kind == "norm_train":
        y, mean, rstd = _norm(s["x"], s["gamma"], s["beta"])
        dx, dgamma, dbeta = _norm_grads(s["dy"], s["x"], s["gamma"], mean, rstd, s["dres"])
        return dict(y=y.to(dt), mean=mean, rstd=rstd, dx=dx.to(dt), dgamma=dgamma.to(dt), dbeta=dbeta.to(dt))
    z = (s["x"].float() + _dropped(s, s["v"].float())).to(dt)
    if kind == "drop":
        return dict(z=z, dv=_dropped(s, s["dy"].float()).to(dt))
    y, mean, rstd = _norm(z, s["gamma"], s["beta"])              # of z as it is handed on
    dz, dgamma, dbeta = _norm_grads(s["dy"], z, s["gamma"], mean, rstd, s["dres"])
    return dict(z=z, y=y.to(dt), mean=mean, rstd=rstd, dz=dz.to(dt), dv=_dropped(s, dz).to(dt), dgamma=dgamma.to(dt), dbeta=dbeta.to(dt))


def _plain_router(s):
    E, k = s["case"]["E"], s["case"]["k"]
    idx = s["topk_idx"].long()
    valid = torch.ones(idx.shape[0], device="cuda") if s["mask"] is None else s["mask"].float()
    ex = torch.exp(s["logits"] - s["logits"].amax(1, keepdim=True))
    p = ex / ex.sum(1, keepdim=True)
    chosen = (idx[:, :, None] == torch.arange(E, device="cuda")).sum(1)                   # [T, E]: 0 or 1
    counts = (chosen * valid[:, None].long()).sum(0)
    n = valid.sum()
    prob_sum = (p * valid[:, None]).double().sum(0)
    f = counts / (k * n).clamp_min(1.0)
    loss = (COEF * E * (f * prob_sum).sum() / n.clamp_min(1.0)).float().view(1)
    out = dict(counts=torch.cat([counts, n.long().view(1)]).int(), prob_sum=prob_sum.float(), loss=loss)
    if s["case"]["kind"] == "balance_train":
        aux = s["dloss"] * (COEF * E / n.clamp_min(1.0)) * p * (f - (p * f).sum(1, keepdim=True)) * valid[:, None]
        w, dw = s["topk_w"], s["dtopk_w"]
        out["dlogits"] = aux.scatter_add(1, idx, w * (dw - (w * dw).sum(1, keepdim=True)))
    return out


def _weights(q, scale):
    """[E, K, N] in 32 bits from codes and scales."""
    E, G, N, _ = q.shape
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
    table = torch.cat([table, -table])
    v = table[torch.stack([q & 15, q >> 4], dim=-1).int()].view(E, G, N, 32)
    return (v * torch.exp2(scale.float() - 127.0)[..., None]).permute(0, 1, 3, 2).reshape(E, G * 32, N)


def _plain_w4(s):
    T, H, I, El, base, k = (s["case"][n] for n in ("T", "H", "I", "E_local", "base", "k"))
    top = torch.sort(s["logits"], dim=1, descending=True, stable=True)
    w = torch.softmax(top.values[:, :k], dim=1)
    share = torch.zeros_like(s["logits"]).scatter(1, top.indices[:, :k], w)[:, base:base + El]     # [T, El]
    h = torch.matmul(s["x"].float(), _weights(s["q_gate_up"], s["s_gate_up"]))                     # [El, T, 2 I]
    a = h[..., :I] * torch.sigmoid(h[..., :I]) * h[..., I:]
    y = torch.matmul(a, _weights(s["q_down"], s["s_down"]))                                        # [El, T, H]
    return dict(out=(y * share.t()[:, :, None]).sum(0).to(torch.bfloat16))


# ---- the framework's operators ----
def _plan(s):
    """Output buffers and workspaces that a program keeps from pass to pass."""
    import paper_2605_23764_amd as moe
    kind, T = s["case"]["kind"], s["case"]["T"]
    b = dict(moe=moe)
    f32 = dict(dtype=torch.float32, device="cuda")
    if kind in ("norm", "norm_train", "drop", "drop_norm"):
        H = s["case"]["H"]
        names = dict(norm=("y",), norm_train=("y", "dx"), drop=("z", "dv"), drop_norm=("z", "y", "dz", "dv"))[kind]
        b.update({n: torch.empty_like(s["x"]) for n in names})
        if kind in ("norm_train", "drop_norm"):
            b.update(mean=torch.empty(T, **f32), rstd=torch.empty(T, **f32), dgamma=torch.empty_like(s["gamma"]),
                     dbeta=torch.empty_like(s["gamma"]), ws=moe.alloc_layer_norm_workspace(T, H))
    elif kind in ("balance", "balance_train"):
        E = s["case"]["E"]
        b.update(counts=torch.empty(E + 1, dtype=torch.int32, device="cuda"), prob_sum=torch.empty(E, **f32),
                 loss=torch.empty(1, **f32), ws=moe.alloc_balance_workspace(T, E))
        if kind == "balance_train":
            b["dlogits"] = torch.empty_like(s["logits"])
    else:
        c = s["case"]
        b["shape"] = moe.make_shape(T, c["H"], c["I"], c["E"], c["E_local"], c["base"], c["k"], torch.bfloat16)
        b.update(ws=moe.alloc_workspace(b["shape"]), out=torch.empty_like(s["x"]))
    return b


def _own(s):
    if "plan" not in s:
        s["plan"] = _plan(s)
    b, kind = s["plan"], s["case"]["kind"]
    moe = b["moe"]
    if kind == "norm":
        moe.moe_layer_norm_forward(s["x"], s["gamma"], s["beta"], EPS, b["y"])
        return dict(y=b["y"])
    if kind == "norm_train":
        moe.moe_layer_norm_forward(s["x"], s["gamma"], s["beta"], EPS, b["y"], b["mean"], b["rstd"])
        moe.moe_layer_norm_backward(s["dy"], s["x"], s["gamma"], b["mean"], b["rstd"], s["dres"], b["dx"], b["dgamma"], b["dbeta"],
                                    b["ws"])
        return {n: b[n] for n in ("y", "mean", "rstd", "dx", "dgamma", "dbeta")}
    if kind == "drop":
        moe.moe_dropout_add_forward(s["v"], s["x"], s["case"]["p"], s["rng"], b["z"])
        moe.moe_dropout_add_backward(s["dy"], s["case"]["p"], s["rng"], b["dv"])
        return dict(z=b["z"], dv=b["dv"])
    if kind == "drop_norm":
        p = s["case"]["p"]
        moe.moe_dropout_add_layer_norm_forward(s["v"], s["x"], p, s["rng"], s["gamma"], s["beta"], EPS, b["z"], b["y"], b["mean"],
                                               b["rstd"])
        moe.moe_dropout_add_layer_norm_backward(s["dy"], b["z"], s["gamma"], b["mean"], b["rstd"], s["dres"], p, s["rng"], b["dz"],
                                                b["dv"], b["dgamma"], b["dbeta"], b["ws"])
        return {n: b[n] for n in ("z", "y", "mean", "rstd", "dz", "dv", "dgamma", "dbeta")}
    if kind == "w4":
        moe.moe_ffn_forward_w4(b["shape"], s["x"], s["logits"], s["q_gate_up"], s["s_gate_up"], s["q_down"], s["s_down"], b["out"],
                               None, b["ws"])
        return dict(out=b["out"])
    moe.moe_balance_forward(s["logits"], s["topk_idx"], s["mask"], COEF, b["counts"], b["prob_sum"], b["loss"], b["ws"])
    out = {n: b[n] for n in ("counts", "prob_sum", "loss")}
    if kind == "balance_train":
        moe.moe_router_backward(s["logits"], s["topk_idx"], s["topk_w"], s["dtopk_w"], s["mask"], COEF, b["counts"], s["dloss"],
                                b["dlogits"])
        out["dlogits"] = b["dlogits"]
    return out


def run(s):
    if own:
        return _own(s)
    kind = s["case"]["kind"]
    return _plain_w4(s) if kind == "w4" else _plain_router(s) if kind.startswith("balance") else _plain_rows(s)


# ---- what a pass cannot do without ----
def work(case):
    T, kind = case["T"], case["kind"]
    if kind in ("norm", "norm_train", "drop", "drop_norm"):
        H, eb = case["H"], 2 if case["dtype"] == "bf16" else 4
        # arrays of T x H read (inputs) and written (outputs), vectors of H, words per row
        arrays, vectors, words, flops = dict(norm=(2, 2, 0, 8), norm_train=(5, 4, 2, 25), drop=(5, 0, 0, 4),
                                             drop_norm=(8, 4, 2, 30))[kind]
        return {"bytes": T * H * eb * arrays + vectors * H * eb + words * T * 4, "flops": T * H * flops}
    E, k = case["E"], case["k"]
    if kind in ("balance", "balance_train"):
        nbytes = T * E * 4 + T * k * 4 + (T if case["masked"] else 0) + 8 * E
        if kind == "balance_train":
            nbytes += T * E * 4 + T * k * 8
        return {"bytes": nbytes, "flops": T * E * (6 if kind == "balance" else 12)}
    H, I, El = case["H"], case["I"], case["E_local"]
    active, rows = El * (1.0 - (1.0 - k / E) ** T), T * k * El / E
    return {"bytes": active * 3 * H * I * (0.5 + 1.0 / 32) + 4 * T * H + 4 * T * E, "flops": 6.0 * rows * H * I}


# ---- the definitions in 64 bits, written apart from the above ----
def _exact_kept(T, H, p, seed, off):
    """Mask from 16-bit halves of products, so that nothing exceeds 63 bits; counters counted off in one line."""
    n8 = -(-H // 8)
    i = torch.arange(T * n8, dtype=torch.int64, device="cuda")
    c = [i % n8, i // n8, torch.full_like(i, off % 2 ** 32), torch.full_like(i, off // 2 ** 32)]
    key = [seed % 2 ** 32, seed // 2 ** 32]

    def product(a, m):
        lo, hi = a * (m % 65536), a * (m // 65536)               # a m = lo + 65536 hi
        low = lo + (hi % 65536) * 65536
        return hi // 65536 + low // 2 ** 32, low % 2 ** 32

    for r in range(10):
        (ah, al), (bh, bl) = product(c[0], 0xD2511F53), product(c[2], 0xCD9E8D57)
        c = [bh ^ c[1] ^ key[0], bl, ah ^ c[3] ^ key[1], al]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    u = torch.empty(T, n8, 8, dtype=torch.int64, device="cuda")
    for j in range(8):
        u[:, :, j] = (c[j // 2] // (65536 if j % 2 else 1) % 65536).view(T, n8)
    return u.view(T, n8 * 8)[:, :H] >= int(p * 65536 + 0.5)


def _exact_rows(case, s):
    T, H, kind, p = case["T"], case["H"], case["kind"], case["p"]
    x = s["x"].double()
    if kind in ("drop", "drop_norm"):
        factor = 1.0
        if p > 0:
            seed, off = (int(v) for v in s["rng"].tolist())
            factor = _exact_kept(T, H, p, seed, off).double() / (1.0 - int(p * 65536 + 0.5) / 65536)
        z = x + s["v"].double() * factor
        if kind == "drop":
            return dict(z=z, dv=s["dy"].double() * factor)
        x = z.to(s["x"].dtype).double()
    g, b = s["gamma"].double(), s["beta"].double()
    mean = x.sum(1) / H
    var = ((x - mean[:, None]) ** 2).sum(1) / H
    rstd = (var + EPS) ** -0.5
    xh = (x - mean[:, None]) * rstd[:, None]
    y = xh * g + b
    if kind == "norm":
        return dict(y=y)
    dy = s["dy"].double()
    t = dy * g
    dx = s["dres"].double() + (t - (t.sum(1) / H)[:, None] - xh * ((t * xh).sum(1) / H)[:, None]) * rstd[:, None]
    out = dict(y=y, mean=mean, rstd=rstd, dgamma=torch.einsum("th,th->h", dy, xh), dbeta=dy.sum(0))
    if kind == "norm_train":
        return dict(out, dx=dx)
    return dict(out, z=z, dz=dx, dv=dx * factor)


def _exact_router(case, s):
    T, E, k = case["T"], case["E"], case["k"]
    valid = torch.ones(T, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"].bool()
    n = int(valid.sum())
    p = torch.softmax(s["logits"].double(), dim=1)
    counts = torch.bincount(s["topk_idx"][valid].long().flatten(), minlength=E)
    prob_sum = p[valid].sum(0)
    f = counts.double() / max(1, k * n)
    out = dict(counts=torch.cat([counts, counts.new_tensor([n])]).int(), prob_sum=prob_sum,
               loss=(COEF * E / max(1, n) * torch.dot(f, prob_sum)).view(1))
    if case["kind"] == "balance_train":
        d = torch.zeros(T, E, dtype=torch.float64, device="cuda")
        pv = p[valid]
        d[valid] = float(s["dloss"]) * COEF * E / max(1, n) * (pv * f - pv * (pv @ f)[:, None])
        w, dw = s["topk_w"].double(), s["dtopk_w"].double()
        dot = (w * dw).sum(1)
        rows = torch.arange(T, device="cuda")
        for j in range(k):
            d[rows, s["topk_idx"][:, j].long()] += w[:, j] * (dw[:, j] - dot)
        out["dlogits"] = d
    return out


def _exact_weights(q, scale):
    """One expert's [K, N] in 64 bits, from the bits of the code: sign, two of exponent (bias 1), one of mantissa."""
    G, N, _ = q.shape
    code = torch.empty(G, N, 32, dtype=torch.int64, device="cuda")
    code[..., 0::2], code[..., 1::2] = (q % 16).long(), (q // 16).long()
    ex, man = code // 2 % 4, code % 2
    mag = torch.where(ex == 0, man * 0.5, (1.0 + 0.5 * man) * 2.0 ** (ex - 1).double())
    v = torch.where(code >= 8, -mag, mag) * (2.0 ** (scale.double() - 127.0))[..., None]
    return v.transpose(1, 2).reshape(G * 32, N)


def _exact_w4(case, s):
    I, El, base, k = (case[n] for n in ("I", "E_local", "base", "k"))
    lg = s["logits"].double()
    order = torch.argsort(lg, dim=1, descending=True, stable=True)[:, :k]
    w = torch.softmax(torch.gather(lg, 1, order), dim=1)
    x = s["x"].double()
    out = torch.zeros_like(x)
    for e in range(El):
        t, j = torch.nonzero(order == base + e, as_tuple=True)
        if t.numel():
            h = x[t] @ _exact_weights(s["q_gate_up"][e], s["s_gate_up"][e])
            a = h[:, :I] / (1.0 + torch.exp(-h[:, :I])) * h[:, I:]
            out.index_add_(0, t, w[t, j][:, None] * (a @ _exact_weights(s["q_down"][e], s["s_down"][e])))
    return dict(out=out)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    return _exact_w4(case, s) if kind == "w4" else _exact_router(case, s) if kind.startswith("balance") else _exact_rows(case, s)
