"""Timed cases of the trainable router and of the update of the experts' weights, in plain torch and through the public entry points.

What a program does with them, and the case kind that stands for it:
  route           routing by scores with everything the layer behind it needs (selection, weights, rows of the experts), inference
  route_train     the same with the gradient of the logits, to which the balance loss's is added, and the step of the balance bias
  project         the router's logits from hidden rows, inference
  project_train   the same with the gradients of the rows, to which the layer's is added, and of the router's weights
  orth            an update made orthogonal by an optimiser of the caller's own
  muon            the whole step: momentum, orthogonal update, weights
"""
from __future__ import annotations

import math

import torch

own = False      # True: run() calls the framework's operators

EPS = 1e-7
STEPS = 5
A, B, C = 3.4445, -4.7750, 2.0315     # of the odd polynomial a s + b s^3 + c s^5
MU, LR, DECAY = 0.95, 0.02, 0.1
RATE = 1e-3


def _route(name, kind, T, E, k, score, groups=1, top_groups=1, renorm=True, scale=1.0, bias=True, E_local=None, base=0):
    return dict(name=name, kind=kind, T=T, E=E, k=k, score=score, groups=groups, top_groups=top_groups, renorm=renorm, scale=scale,
                bias=bias, E_local=E_local or E, base=base)


def _project(name, kind, T, H, E, dtype="bf16"):
    return dict(name=name, kind=kind, T=T, H=H, E=E, dtype=dtype)


def _update(name, kind, n, M, N, dtype="bf16"):
    return dict(name=name, kind=kind, B=n, M=M, N=N, dtype=dtype)


def listed():
    return [
        # one token of a decode step: sigmoid scores, eight groups, 32 of 256 experts on this GPU
        _route("route_1_large", "route", 1, 256, 8, "sigmoid", 8, 4, True, 2.5, E_local=32, base=64),
        # a serving batch of a mid-size softmax router without groups
        _route("route_200_softmax", "route", 200, 60, 6, "softmax", renorm=False, bias=False),
        # a training step's router at the headline shape
        _route("route_train_8192_large", "route_train", 8192, 256, 8, "sigmoid", 8, 4, True, 2.5, E_local=32),
        # many tokens, few experts in groups, weights as they are, an odd count
        _route("route_train_30001", "route_train", 30001, 64, 6, "softmax", 4, 2, False, 1.5, E_local=16, base=16),
        # one token's logits: the weights' trip through the chip
        _project("project_1_large", "project", 1, 7168, 256),
        # a training step's projection at the headline shape
        _project("project_train_8192_large", "project_train", 8192, 7168, 256),
        # fp32 storage, rows that no vector divides, few experts
        _project("project_train_1500_odd_f32", "project_train", 1500, 1001, 24, "f32"),
        # one small matrix: launches and latency
        _update("orth_1_small", "orth", 1, 200, 330),
        # four experts' down projections of a mid-size layer, fp32 storage
        _update("orth_4_mid_f32", "orth", 4, 1408, 2048, "f32"),
        # ten experts of an odd width, fp32 storage
        _update("muon_10_odd_f32", "muon", 10, 704, 1088, "f32"),
        # every expert's gate and up projections of a mid-size layer
        _update("muon_16_mid", "muon", 16, 2048, 2816),
        # four experts' gate and up projections of the large layer
        _update("muon_4_large", "muon", 4, 7168, 4096),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["route", "route_train", "route_train", "project", "project_train", "project_train", "orth", "orth", "muon", "muon"])
    if kind in ("route", "route_train"):
        E = rng.choice([8, 16, 24, 60, 64, 128, 160, 256])
        groups = rng.choice([g for g in (1, 1, 2, 4, 8) if E % g == 0])
        top = rng.randint(1, groups)
        E_local = rng.choice([e for e in (4, 8, 10, 16, 32, E) if e <= E])
        return dict(kind=kind, T=_log_int(rng, 1 if kind == "route" else 32, 32768), E=E, k=rng.randint(1, min(8, top * (E // groups))),
                    score=rng.choice(["sigmoid", "softmax"]), groups=groups, top_groups=top, renorm=rng.random() < 0.5,
                    scale=rng.choice([1.0, 1.5, 2.5]), bias=rng.random() < 0.7, E_local=E_local, base=rng.randint(0, E - E_local))
    if kind in ("project", "project_train"):
        H = 64 * _log_int(rng, 1, 112) if rng.random() < 0.7 else _log_int(rng, 33, 7168)
        return dict(kind=kind, T=_log_int(rng, 1 if kind == "project" else 16, 8192), H=H, E=rng.choice([8, 16, 24, 60, 64, 128, 160, 256]),
                    dtype="f32" if rng.random() < 0.35 else "bf16")
    M, N = ((64 * _log_int(rng, 1, 64) if rng.random() < 0.6 else _log_int(rng, 24, 4096)) for _ in range(2))
    short, long = min(M, N), max(M, N)
    most = int(5e11 / (3.0 * short * short * long + short ** 3))          # matrices whose products stay below the largest case's
    return dict(kind=kind, B=_log_int(rng, 1, max(1, min(16, most))), M=M, N=N, dtype="f32" if rng.random() < 0.35 else "bf16")


# ---- inputs ----
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _spectrum(n, M, N, g, size):
    """Matrices with a few strong directions over a broad rest, as momentum has them."""
    r = max(1, min(M, N) // 16)
    strong = torch.randn(n, M, r, generator=g, device="cuda") @ torch.randn(n, r, N, generator=g, device="cuda")
    return (strong * r ** -0.5 + torch.randn(n, M, N, generator=g, device="cuda")) * size


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    kind = case["kind"]
    s = dict(case=case)
    if kind in ("route", "route_train"):
        T, E, k = case["T"], case["E"], case["k"]
        s["logits"] = torch.randn(T, E, generator=g, device="cuda") + 0.5 * torch.randn(E, generator=g, device="cuda")
        s["bias"] = 0.05 * torch.randn(E, generator=g, device="cuda") if case["bias"] else None
        if kind == "route_train":
            s["dtopk_w"] = torch.randn(T, k, generator=g, device="cuda") / T
            s["dbalance"] = 0.01 * torch.randn(T, E, generator=g, device="cuda") / T      # the balance loss's gradient
            mean = max(1, T * k // E)                                                     # selections of every rank's tokens
            s["counts"] = torch.randint(0, 2 * mean + 1, (E + 1,), generator=g, device="cuda").to(torch.int32)
        return s
    if kind in ("project", "project_train"):
        T, H, E, dt = case["T"], case["H"], case["E"], _dtype(case)
        s["x"] = torch.randn(T, H, generator=g, device="cuda").to(dt)
        s["w"] = torch.randn(H, E, generator=g, device="cuda") * H ** -0.5
        if kind == "project_train":
            s["dlogits"] = torch.randn(T, E, generator=g, device="cuda")
            s["dlayer"] = torch.randn(T, H, generator=g, device="cuda").to(dt)            # the layer's gradient of the rows
        return s
    n, M, N, dt = case["B"], case["M"], case["N"], _dtype(case)
    if kind == "orth":
        s["u"] = _spectrum(n, M, N, g, 1e-3).to(dt)
        return s
    s["g"] = torch.empty(n, M, N, dtype=dt, device="cuda")
    s["m"] = torch.empty(n, M, N, device="cuda")
    s["w"] = torch.empty(n, M, N, dtype=dt, device="cuda")
    for e in range(n):                                                                    # one at a time: they are large
        s["m"][e] = _spectrum(1, M, N, g, 1e-3)[0]
        s["g"][e] = 0.05 * s["m"][e] + 2e-4 * torch.randn(M, N, generator=g, device="cuda")
        s["w"][e] = torch.randn(M, N, generator=g, device="cuda") * M ** -0.5
    return s


# ---- the plain form ----
def _scores(c, logits):
    """In 64 bits: the selection is decided at borders between neighbouring scores."""
    l = logits.double()
    if c["score"] == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-l))
    e = torch.exp(l - l.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True)


def _plain_route(s):
    c = s["case"]
    T, E, k, G, El, base = (c[n] for n in ("T", "E", "k", "groups", "E_local", "base"))
    dev = s["logits"].device
    p = _scores(c, s["logits"])
    key = p if s["bias"] is None else p + s["bias"].double()
    if G > 1:
        per = key.view(T, G, E // G)
        best = torch.sort(per, dim=2, descending=True).values[:, :, :2].sum(2)
        keep = torch.sort(best, dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        alive = torch.zeros(T, G, dtype=torch.bool, device=dev).scatter(1, keep, True)
        key = torch.where(alive[:, :, None], per, -math.inf).reshape(T, E)
    idx = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :k]
    ps = torch.gather(p, 1, idx)
    share = ps / ps.sum(1, keepdim=True) if c["renorm"] else ps
    # rows of the local experts: by expert, then by token
    expert = torch.where((idx >= base) & (idx < base + El), idx - base, El).flatten()
    order = torch.sort(expert, stable=True).indices
    sorted_expert = expert[order]
    local = sorted_expert < El
    row_of = torch.empty_like(order).scatter(0, order, torch.where(local, torch.arange(T * k, device=dev), -1))
    counts = (expert[:, None] == torch.arange(El, device=dev)).sum(0)
    most = T * min(k, El)
    tables = [torch.where(local, v, -1)[:most].int() for v in (order // k, order % k)]
    out = dict(topk_idx=idx.int(), topk_w=(share * c["scale"]).float(), counts=counts.int(),
               offsets=torch.cat([counts.new_zeros(1), counts.cumsum(0)]).int(), row_of=row_of.view(T, k).int(), token_of=tables[0],
               slot_of=tables[1])
    if c["kind"] == "route_train":
        dw = s["dtopk_w"].double() * c["scale"]
        t = dw - (share * dw).sum(1, keepdim=True) if c["renorm"] else dw
        if c["score"] == "sigmoid":
            d = torch.zeros_like(p).scatter(1, idx, share * t * (1.0 - ps))
        else:
            d = torch.zeros_like(p).scatter(1, idx, share * t)
            d = d if c["renorm"] else d - p * (ps * dw).sum(1, keepdim=True)
        out["dlogits"] = (s["dbalance"].double() + d).float()
        if s["bias"] is not None:
            n = s["counts"][:E].long()
            out["bias"] = s["bias"] + RATE * torch.sign(n.sum() - E * n).float()
    return out


def _plain_project(s):
    x, dt = s["x"].float(), s["x"].dtype
    out = dict(logits=torch.matmul(x, s["w"]))
    if s["case"]["kind"] == "project_train":
        out["dx"] = (s["dlayer"].float() + torch.matmul(s["dlogits"], s["w"].t())).to(dt)
        out["dw"] = torch.matmul(x.t(), s["dlogits"])
    return out


def _polynomial(u):
    """Of the singular values of u [n, M, N] over its norm: STEPS times a s + b s^3 + c s^5."""
    wide = u.shape[1] <= u.shape[2]
    x = u if wide else u.transpose(1, 2).contiguous()
    norm = torch.sqrt((x.double() * x.double()).sum((1, 2), keepdim=True)).float()
    x = x / (norm + EPS)
    for _ in range(STEPS):
        a = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = A * x + torch.matmul(B * a + C * torch.matmul(a, a), x)
    return x if wide else x.transpose(1, 2)


def _update_scale(c):
    return max(1.0, c["M"] / c["N"]) ** 0.5


def _plain_update(s):
    c = s["case"]
    if c["kind"] == "orth":
        return dict(o=_polynomial(s["u"].float()).to(s["u"].dtype).contiguous())
    g = s["g"].float()
    m = MU * s["m"] + g
    o = _polynomial(g + MU * m)
    return dict(m=m, w=(s["w"].float() * (1.0 - LR * DECAY) - LR * _update_scale(c) * o).to(s["w"].dtype))


# ---- the framework's operators ----
def _plan(s):
    """Handles, output buffers and workspaces that a program keeps from pass to pass."""
    import paper_2605_23764_amd as moe
    c, kind = s["case"], s["case"]["kind"]
    b = dict(moe=moe)
    if kind in ("route", "route_train"):
        b["scores"] = moe.make_scores(c["score"], c["groups"], c["top_groups"], c["renorm"], c["scale"])
        b["shape"] = moe.make_shape(c["T"], 64, 64, c["E"], c["E_local"], c["base"], c["k"], torch.bfloat16)
        b["saved"], b["ws"] = moe.alloc_saved(b["shape"], keep_xp=False), moe.alloc_workspace(b["shape"])
        b["saved"].token_of.fill_(-1)            # rows behind the last stay as they are
        b["saved"].slot_of.fill_(-1)
        if kind == "route_train":
            b["dlogits"] = torch.empty_like(s["logits"])
            b["bias"] = None if s["bias"] is None else torch.empty_like(s["bias"])
    elif kind in ("project", "project_train"):
        T, H, E = c["T"], c["H"], c["E"]
        b.update(ws=moe.alloc_router_project_workspace(T, H, E), logits=torch.empty(T, E, device="cuda"))
        if kind == "project_train":
            b.update(dx=torch.empty_like(s["x"]), dw=torch.empty_like(s["w"]))
    else:
        b["ws"] = moe.alloc_muon_workspace(c["B"], c["M"], c["N"], _dtype(c))
        if kind == "orth":
            b["o"] = torch.empty_like(s["u"])
        else:
            b.update(m=torch.empty_like(s["m"]), w=torch.empty_like(s["w"]))
    return b


def _own(s):
    if "plan" not in s:
        s["plan"] = _plan(s)
    b, c, kind = s["plan"], s["case"], s["case"]["kind"]
    moe = b["moe"]
    if kind in ("route", "route_train"):
        sv = b["saved"]
        moe.moe_route_scores(b["shape"], b["scores"], s["logits"], s["bias"], sv, b["ws"])
        out = {n: getattr(sv, n) for n in ("topk_idx", "topk_w", "counts", "offsets", "row_of", "token_of", "slot_of")}
        if kind == "route_train":
            moe.moe_route_scores_backward(b["scores"], s["logits"], sv.topk_idx, s["dtopk_w"], s["dbalance"], b["dlogits"])
            out["dlogits"] = b["dlogits"]
            if s["bias"] is not None:
                moe.moe_bias_update(s["counts"], RATE, s["bias"], b["bias"])
                out["bias"] = b["bias"]
        return out
    if kind in ("project", "project_train"):
        moe.moe_router_project(s["x"], s["w"], b["logits"], b["ws"])
        if kind == "project":
            return dict(logits=b["logits"])
        moe.moe_router_project_backward(s["dlogits"], s["x"], s["w"], s["dlayer"], b["dx"], b["dw"], b["ws"])
        return {n: b[n] for n in ("logits", "dx", "dw")}
    if kind == "orth":
        moe.moe_orthogonalize(s["u"], b["o"], b["ws"], steps=STEPS, eps=EPS)
        return dict(o=b["o"])
    moe.moe_muon_step(s["g"], s["m"], s["w"], b["m"], b["w"], b["ws"], lr=LR, mu=MU, nesterov=True, weight_decay=DECAY,
                      scale=_update_scale(c), steps=STEPS, eps=EPS)
    return dict(m=b["m"], w=b["w"])


def run(s):
    if own:
        return _own(s)
    kind = s["case"]["kind"]
    return _plain_route(s) if kind.startswith("route") else _plain_project(s) if kind.startswith("project") else _plain_update(s)


# ---- what a pass cannot do without ----
def work(case):
    kind = case["kind"]
    if kind in ("route", "route_train"):
        T, E, k = case["T"], case["E"], case["k"]
        rows = T * k * case["E_local"] / E
        nbytes = T * E * 4 + T * k * 12 + rows * 8 + 8 * case["E_local"]
        if kind == "route_train":
            nbytes += T * E * 8 + T * k * 4 + 12 * E
        return {"bytes": nbytes, "flops": T * E * (10 if kind == "route" else 16)}
    if kind in ("project", "project_train"):
        T, H, E, eb = case["T"], case["H"], case["E"], 2 if case["dtype"] == "bf16" else 4
        nbytes, flops = T * H * eb + H * E * 4 + T * E * 4, 2.0 * T * H * E
        if kind == "project_train":
            nbytes, flops = nbytes + T * H * eb * 2 + H * E * 4 + T * E * 4, 3 * flops
        return {"bytes": nbytes, "flops": flops}
    n, M, N, eb = case["B"], case["M"], case["N"], 2 if case["dtype"] == "bf16" else 4
    short, long = min(M, N), max(M, N)
    per = 2 * eb if kind == "orth" else 3 * eb + 8
    # the two symmetric products count half
    return {"bytes": n * M * N * per, "flops": float(n) * STEPS * (3.0 * short * short * long + float(short) ** 3)}


# ---- the definitions in 64 bits, written apart from the above ----
def _exact_route(c, s):
    T, E, k, G = c["T"], c["E"], c["k"], c["groups"]
    l = s["logits"].double()
    p = torch.sigmoid(l) if c["score"] == "sigmoid" else torch.softmax(l, dim=1)
    key = p.clone() if s["bias"] is None else p + s["bias"].double()
    if G > 1:
        size = E // G
        total = torch.stack([torch.topk(key[:, i * size:(i + 1) * size], min(2, size), dim=1).values.sum(1) for i in range(G)], dim=1)
        stay = torch.zeros(T, G, dtype=torch.bool, device="cuda")
        for _ in range(c["top_groups"]):
            at = total.argmax(1, keepdim=True)
            stay.scatter_(1, at, True)
            total.scatter_(1, at, -math.inf)
        key[~stay.repeat_interleave(size, dim=1)] = -math.inf
    idx = torch.empty(T, k, dtype=torch.int64, device="cuda")
    for j in range(k):
        first = (key == key.max(1, keepdim=True).values).to(torch.int8).argmax(1)
        idx[:, j] = first
        key[torch.arange(T, device="cuda"), first] = -math.inf
    ps = torch.gather(p, 1, idx)
    total = ps.sum(1, keepdim=True) if c["renorm"] else torch.ones_like(ps[:, :1])
    w = c["scale"] * ps / total
    El, base = c["E_local"], c["base"]
    row_of = torch.full((T, k), -1, dtype=torch.int64, device="cuda")
    token_of, slot_of = (torch.full((T * min(k, El),), -1, dtype=torch.int64, device="cuda") for _ in range(2))
    offsets = [0]
    for e in range(El):
        t, j = torch.nonzero(idx == base + e, as_tuple=True)
        r = torch.arange(offsets[-1], offsets[-1] + t.numel(), device="cuda")
        row_of[t, j], token_of[r], slot_of[r] = r, t, j
        offsets.append(offsets[-1] + t.numel())
    offsets = torch.tensor(offsets, device="cuda")
    out = dict(topk_idx=idx.int(), topk_w=w, counts=(offsets[1:] - offsets[:-1]).int(), offsets=offsets.int(), row_of=row_of.int(),
               token_of=token_of.int(), slot_of=slot_of.int())
    if c["kind"] == "route_train":
        # the chain rule, step by step: weights -> scores -> logits
        dw = s["dtopk_w"].double()
        dps = c["scale"] * (dw / total - ((dw * ps).sum(1, keepdim=True) / total ** 2 if c["renorm"] else 0.0))
        dp = torch.zeros_like(p).scatter_add(1, idx, dps)
        d = dp * p * torch.sigmoid(-l) if c["score"] == "sigmoid" else p * (dp - (p * dp).sum(1, keepdim=True))
        out["dlogits"] = d + s["dbalance"].double()
        if s["bias"] is not None:
            n = s["counts"][:E].double()
            out["bias"] = s["bias"].double() + RATE * torch.sign(n.mean() - n)
    return out


def _exact_project(c, s):
    x, w = s["x"].double(), s["w"].double()
    out = dict(logits=x @ w)
    if c["kind"] == "project_train":
        d = s["dlogits"].double()
        out.update(dx=s["dlayer"].double() + d @ w.t(), dw=x.t() @ d)
    return out


def _exact_update(c, s):
    n = c["B"]

    def polynomial(u):
        """One matrix; Horner's form on the side of the columns or rows that is shorter."""
        x = u / (torch.linalg.vector_norm(u) + EPS)
        eye = torch.eye(min(u.shape), dtype=torch.float64, device="cuda")
        for _ in range(STEPS):
            if x.shape[0] <= x.shape[1]:
                q = x @ x.t()
                x = (A * eye + (B * eye + C * q) @ q) @ x
            else:
                q = x.t() @ x
                x = x @ (A * eye + q @ (B * eye + C * q))
        return x

    if c["kind"] == "orth":
        return dict(o=torch.stack([polynomial(s["u"][e].double()) for e in range(n)]))
    m, w = [], []
    for e in range(n):
        g = s["g"][e].double()
        m.append(s["m"][e].double() * MU + g)
        o = polynomial(m[-1] * MU + g)
        w.append(s["w"][e].double() - LR * (DECAY * s["w"][e].double() + max(1.0, c["M"] / c["N"]) ** 0.5 * o))
    return dict(m=torch.stack(m), w=torch.stack(w))


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    return _exact_route(case, s) if kind.startswith("route") else _exact_project(case, s) if kind.startswith("project") else _exact_update(case, s)
