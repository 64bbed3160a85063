"""Row operators at the largest row counts that a call takes: T is 31 bits, and rows of a few elements still fit into memory."""
import numpy as np
import pytest
import torch

import paper_2605_23764_amd as moe
from block_common import f64
from oracle import block_oracle as bo

pytestmark = pytest.mark.gpu

LAST = 2 ** 31 - 1


def _kept(t, seed, offset, thr):
    """Element (t, 0): kept if the low half of the generator's first word is at least thr."""
    word = bo.philox4x32_10([np.zeros_like(t), t, np.full_like(t, offset % 2 ** 32), np.full_like(t, offset >> 32)], [seed % 2 ** 32, seed >> 32])[0]
    return (word & np.uint64(0xFFFF)).astype(np.int64) >= thr


@pytest.mark.parametrize("T", [LAST - 31, LAST - 30, LAST])
def test_dropout_of_all_rows(T):
    """Counted in groups of 32 rows: the count of the last groups may not leave 31 bits."""
    print(f"dropout T={T} H=1", flush=True)
    v = torch.arange(T % 1024, T % 1024 + 256, device="cuda", dtype=torch.int16).to(torch.bfloat16).repeat(T // 256 + 1)[:T].view(T, 1)
    out = torch.full_like(v, -1.0)
    moe.moe_dropout_add_forward(v, None, 0.0, None, out)
    assert torch.equal(out, v)
    out.fill_(-1.0)
    rng = torch.tensor([2 ** 35 + 9, 2 ** 34 + 4], dtype=torch.int64, device="cuda")
    moe.moe_dropout_add_backward(v, 0.5, rng, out)
    for lo, hi in ((0, 512), (T // 2, T // 2 + 512), (T - 512, T)):
        want = np.where(_kept(np.arange(lo, hi), 2 ** 35 + 9, 2 ** 34 + 4, 32768), 2 * f64(v[lo:hi, 0]), 0.0)   # exact: twice the value
        np.testing.assert_array_equal(f64(out[lo:hi, 0]), want)
    assert not (out == -1.0).any()


def test_layer_norm_of_all_rows():
    """Rows of one element: y is beta, the gradient what came along the residual path."""
    print(f"layer norm T={LAST} H=1", flush=True)
    x = torch.arange(256, device="cuda", dtype=torch.int16).to(torch.bfloat16).repeat(LAST // 256 + 1)[:LAST].view(LAST, 1)
    one, beta = torch.ones(1, dtype=torch.bfloat16, device="cuda"), torch.full((1,), 0.75, dtype=torch.bfloat16, device="cuda")
    y = torch.full_like(x, -1.0)
    mean, rstd = (torch.full((LAST,), -1.0, device="cuda") for _ in range(2))
    moe.moe_layer_norm_forward(x, one, beta, 1.0, y, mean, rstd)
    assert (y == 0.75).all() and (rstd == 1.0).all() and torch.equal(mean[-4096:], x[-4096:, 0].float())
    dx = torch.full_like(x, -1.0)
    moe.moe_layer_norm_backward(y, x, one, mean, rstd, x, dx, None, None, None)
    assert torch.equal(dx, x)
