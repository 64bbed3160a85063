"""More values than 31 bits count, in groups of matrices: the last ones are what they are alone."""
import pytest
import torch

import paper_2605_23764_amd as moe

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("master", [False, True], ids=["weights", "master"])
def test_more_than_31_bits_of_values(master):
    n, M, N = 66001, 128, 256
    print(f"muon_step {n} x {M} x {N}, master {master}", flush=True)
    bf = torch.bfloat16
    g, w = torch.zeros(n, M, N, dtype=bf, device="cuda"), torch.zeros(n, M, N, dtype=bf, device="cuda")
    m, top = torch.zeros(n, M, N, device="cuda"), torch.zeros(n, M, N, device="cuda") if master else None
    gen = torch.Generator("cuda").manual_seed(0)
    at = [0, 1, 32767, 32768, 65535, 65536, n - 2, n - 1]
    for e in at:
        g[e], w[e] = (torch.randn(M, N, generator=gen, device="cuda").to(bf) for _ in range(2))
        m[e] = torch.randn(M, N, generator=gen, device="cuda")
        if master:
            top[e] = w[e].float()
    alone = [(g[e:e + 1].clone(), m[e:e + 1].clone(), w[e:e + 1].clone(), top[e:e + 1].clone() if master else None) for e in at]
    kw = dict(lr=0.3, mu=0.9, weight_decay=0.1)
    moe.moe_muon_step(g, m, None if master else w, m, w, moe.alloc_muon_workspace(n, M, N, bf), master=top, **kw)
    ws = moe.alloc_muon_workspace(1, M, N, bf)
    for e, (g1, m1, w1, t1) in zip(at, alone):
        moe.moe_muon_step(g1, m1, None if master else w1, m1, w1, ws, master=t1, **kw)
        assert torch.equal(w[e], w1[0]) and torch.equal(m[e], m1[0]), e
        if master:
            assert torch.equal(top[e], t1[0]), e
    assert not w[2].any() and not m[40000].any() and not w[n - 3].any()          # zeros stay zeros
