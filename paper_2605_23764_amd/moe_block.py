"""One pre-norm MoE block of a transformer on the operators of this package: a training step, and a decode step with 4-bit experts.

    y = layer_norm(x);  logits = y W_router;  m = MoE-FFN(y, logits);  z = x + dropout(m);  out = next block's layer_norm(z)

with the balance loss of the router.  Everything but the router's small projection (a library product) runs in the HIP library; the caller
owns every buffer, as everywhere here.  With scores (make_scores) the router is another: its projection runs in the library too, experts
are selected by sigmoid or softmax scores and a bias that moves towards balance.  update() is the optimiser's step of the experts: momentum
and orthogonal updates, of gate and up apart or as one matrix.

    python -m paper_2605_23764_amd.moe_block [--tokens 4096 --hidden 2048 --width 1408 --experts 16 --top-k 4 --dropout 0.1]
                                             [--scores sigmoid --groups 4 --top-groups 2]
"""
from __future__ import annotations

import argparse
import time

import torch

from . import binding as moe


class MoeBlock:
    """Weights and buffers of one block for T tokens, every expert on this GPU."""

    def __init__(self, T, H, I, E, k, dtype=torch.bfloat16, p=0.1, coef=0.01, eps=1e-5, seed=0, device="cuda",
                 scores=None, rate=1e-3):
        self.T, self.H, self.E, self.k, self.p, self.coef, self.eps = T, H, E, k, p, coef, eps
        g = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, scale=1.0):
            return (torch.randn(*shape, generator=g, device=device) * scale).to(dtype)
        self.w_router = torch.randn(H, E, generator=g, device=device) * H ** -0.5
        self.w_gate_up, self.w_down = normal(E, H, 2 * I, scale=H ** -0.5), normal(E, I, H, scale=I ** -0.5)
        self.gamma, self.gamma_next = (torch.ones(H, dtype=dtype, device=device) for _ in range(2))
        self.beta, self.beta_next = (torch.zeros(H, dtype=dtype, device=device) for _ in range(2))
        self.rng = torch.tensor([seed, 0], dtype=torch.int64, device=device)      # {seed, offset}: the offset moves on with every step
        self.shape = moe.make_shape(T, H, I, E, E, 0, k, dtype)
        self.saved = moe.alloc_saved(self.shape, store_h1=True, keep_xp=False)
        self.ws = moe.alloc_workspace(self.shape, device, backward=True)
        self.ws_norm, self.ws_balance = moe.alloc_layer_norm_workspace(T, H, device), moe.alloc_balance_workspace(T, E, device)

        def rows():
            return torch.empty(T, H, dtype=dtype, device=device)

        def f32(*shape):
            return torch.empty(*shape, dtype=torch.float32, device=device)
        self.y, self.m, self.z, self.out = rows(), rows(), rows(), rows()
        self.mean, self.rstd, self.mean_next, self.rstd_next = (f32(T) for _ in range(4))
        self.counts = torch.empty(E + 1, dtype=torch.int32, device=device)
        self.prob_sum, self.loss, self.dtopk_w, self.dlogits = f32(E), f32(1), f32(T, k), f32(T, E)
        self.dx, self.dz, self.dm, self.dy = rows(), rows(), rows(), rows()
        self.dw_gate_up, self.dw_down = torch.empty_like(self.w_gate_up), torch.empty_like(self.w_down)
        self.dgamma, self.dbeta, self.dgamma_next, self.dbeta_next = (torch.empty_like(self.gamma) for _ in range(4))
        self.dw_router = torch.empty_like(self.w_router)
        self.blocks = self.momentum = None
        self.scores, self.rate = scores, rate                                       # None: softmax over the k selected logits, no bias
        if scores is not None:
            self.bias, self.logits = torch.zeros(E, device=device), f32(T, E)
            self.ws_project = moe.alloc_router_project_workspace(T, H, E, device)

    def forward(self, x, mask=None):
        """(out, z): the next block's normalised input and its residual stream; self.loss is the balance loss.  mask [T]: 0 marks padding."""
        self.x, self.mask = x, mask
        moe.moe_layer_norm_forward(x, self.gamma, self.beta, self.eps, self.y, self.mean, self.rstd)
        if self.scores is None:
            self.logits = self.y.float() @ self.w_router
            moe.moe_ffn_forward(self.shape, self.y, self.logits, self.w_gate_up, self.w_down, self.m, self.saved, self.ws)
        else:
            moe.moe_router_project(self.y, self.w_router, self.logits, self.ws_project)
            moe.moe_route_scores(self.shape, self.scores, self.logits, self.bias, self.saved, self.ws)
            moe.moe_dispatch_to_combine(self.shape, self.y, self.w_gate_up, self.w_down, self.m, self.saved, self.ws)
        moe.moe_balance_forward(self.logits, self.saved.topk_idx, mask, self.coef, self.counts, self.prob_sum, self.loss, self.ws_balance)
        moe.moe_dropout_add_layer_norm_forward(self.m, x, self.p, self.rng, self.gamma_next, self.beta_next, self.eps, self.z, self.out,
                                               self.mean_next, self.rstd_next)
        return self.out, self.z

    def backward(self, dout, dz):
        """Gradient of x from those of out and z, and of the balance loss; the weights' are left in the block's d* buffers."""
        moe.moe_dropout_add_layer_norm_backward(dout, self.z, self.gamma_next, self.mean_next, self.rstd_next, dz, self.p, self.rng, self.dz,
                                                self.dm, self.dgamma_next, self.dbeta_next, self.ws_norm)
        moe.moe_ffn_backward(self.shape, self.dm, self.y, self.w_gate_up, self.w_down, self.saved, self.dy, self.dw_gate_up, self.dw_down,
                             self.dtopk_w, self.ws)
        if self.scores is None:
            moe.moe_router_backward(self.logits, self.saved.topk_idx, self.saved.topk_w, self.dtopk_w, self.mask, self.coef, self.counts, None,
                                    self.dlogits)
            torch.mm(self.y.float().t(), self.dlogits, out=self.dw_router)
            self.dy += (self.dlogits @ self.w_router.t()).to(self.dy.dtype)
        else:
            moe.moe_router_backward(self.logits, self.saved.topk_idx, None, None, self.mask, self.coef, self.counts, None, self.dlogits)
            moe.moe_route_scores_backward(self.scores, self.logits, self.saved.topk_idx, self.dtopk_w, self.dlogits, self.dlogits)
            moe.moe_router_project_backward(self.dlogits, self.y, self.w_router, self.dy, self.dy, self.dw_router, self.ws_project)
        moe.moe_layer_norm_backward(self.dy, self.x, self.gamma, self.mean, self.rstd, self.dz, self.dx, self.dgamma, self.dbeta,
                                    self.ws_norm)
        return self.dx

    def step(self, x, dout, dz, mask=None):
        """One training step's forward and backward, with a new dropout mask."""
        self.rng[1] += 1
        self.forward(x, mask)
        return self.backward(dout, dz)

    def update(self, lr=0.02, mu=0.95, weight_decay=0.0, scale=1.0, apart=False):
        """After step(): the experts' weights by momentum and orthogonal updates; with scores the bias too.

        apart: each expert's gate and up matrices [H, I] by themselves, else [H, 2I] as one matrix, as they are stored; w_down [I, H] by itself.
        scale: of the orthogonal matrices, or "fan": max(1, fan_out / fan_in)^0.5 of each (weights are [in, out]).  Momentum belongs to the form
        of the first call."""
        E, H, I = self.E, self.H, self.shape.I
        halves = (2 * E, H, I)
        if self.momentum is None:
            sizes = (halves if apart else tuple(self.w_gate_up.shape), tuple(self.w_down.shape))
            self.momentum = [torch.zeros(n, device=self.w_down.device) for n in sizes]
            self.ws_update = [moe.alloc_muon_workspace(*n, self.w_down.dtype, self.w_down.device) for n in sizes]
            if apart:
                self.w_halves, self.dw_halves = (torch.empty(halves, dtype=self.w_down.dtype, device=self.w_down.device) for _ in range(2))
        elif (self.momentum[0].shape == halves) != bool(apart):
            raise ValueError("apart: the momentum is that of the other form")
        w1, dw1 = self.w_gate_up, self.dw_gate_up
        if apart:                                                    # [E, H, 2, I] with gate and up in front
            w1, dw1 = self.w_halves, self.dw_halves
            for half, whole in ((w1, self.w_gate_up), (dw1, self.dw_gate_up)):
                half.view(2, E, H, I).copy_(whole.view(E, H, 2, I).permute(2, 0, 1, 3))
        for w, dw, m, ws in zip((w1, self.w_down), (dw1, self.dw_down), self.momentum, self.ws_update):
            fan_in, fan_out = w.shape[1:]
            s = max(1.0, fan_out / fan_in) ** 0.5 if scale == "fan" else scale
            moe.moe_muon_step(dw, m, w, m, w, ws, lr=lr, mu=mu, weight_decay=weight_decay, scale=s)
        if apart:
            self.w_gate_up.view(E, H, 2, I).copy_(w1.view(2, E, H, I).permute(1, 2, 0, 3))
        if self.scores is not None:
            moe.moe_bias_update(self.counts, self.rate, self.bias, self.bias)

    def quantize(self):
        """The experts as 4-bit blocks, for decode()."""
        self.blocks = []
        for w in (self.w_gate_up, self.w_down):
            q, scale = moe.alloc_w4(*w.shape, device=w.device)
            moe.moe_quantize_w4(w, q, scale)
            self.blocks += [q, scale]

    def decode(self, x):
        """x + the layer's output for up to T tokens in bfloat16, experts in 4 bits, nothing dropped."""
        T, dev = x.shape[0], x.device
        y, m, z = (torch.empty_like(x) for _ in range(3))
        moe.moe_layer_norm_forward(x, self.gamma, self.beta, self.eps, y)
        shape = moe.make_shape(T, self.H, self.shape.I, self.E, self.E, 0, self.k, x.dtype)
        ws = torch.empty(moe.moe_ffn_workspace_bytes(shape)[0], dtype=torch.uint8, device=dev)
        if self.scores is None:
            moe.moe_ffn_forward_w4(shape, y, y.float() @ self.w_router, *self.blocks, m, None, ws)
        else:
            logits, saved = torch.empty(T, self.E, device=dev), moe.alloc_saved(shape, dev, keep_xp=False)
            moe.moe_router_project(y, self.w_router, logits, moe.alloc_router_project_workspace(T, self.H, self.E, dev))
            moe.moe_route_scores(shape, self.scores, logits, self.bias, saved, ws)
            moe.moe_dispatch_to_combine_w4(shape, y, *self.blocks, m, saved, ws)
        moe.moe_dropout_add_forward(m, x, 0.0, None, z)
        return z


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("tokens", 4096), ("hidden", 2048), ("width", 1408), ("experts", 16), ("top-k", 4), ("steps", 20)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--dropout", type=float, default=0.1)
    ap.add_argument("--scores", choices=("sigmoid", "softmax"), help="route by scores with a balance bias")
    for name in ("groups", "top-groups"):
        ap.add_argument("--" + name, type=int, default=1)
    a = ap.parse_args()
    scores = moe.make_scores(a.scores, a.groups, a.top_groups) if a.scores else None
    block = MoeBlock(a.tokens, a.hidden, a.width, a.experts, a.top_k, p=a.dropout, scores=scores)
    x, dout, dz = (torch.randn(a.tokens, a.hidden, device="cuda").to(torch.bfloat16) for _ in range(3))

    def timed(what, fn):
        for _ in range(3):
            fn()
        torch.cuda.synchronize()
        t = time.perf_counter()
        for _ in range(a.steps):
            fn()
        torch.cuda.synchronize()
        print(f"{what}: {(time.perf_counter() - t) / a.steps * 1e6:.1f} us", flush=True)

    timed(f"training step, {a.tokens} tokens", lambda: block.step(x, dout, dz))
    print(f"balance loss {block.loss.item():.5f} ({block.coef} if even), busiest expert {block.counts[:-1].max().item()} of "
          f"{a.tokens * a.top_k // a.experts} selections on average")
    timed("update of the experts, gate and up apart", lambda: block.update(scale="fan", apart=True))
    block.quantize()
    for n in (1, 32):
        timed(f"decode step, {n} tokens, 4-bit experts", lambda: block.decode(x[:n]))


if __name__ == "__main__":
    main()
