"""The layer operators at the ends of what they take: rows of nearly 2^31 columns, and more work items than one dimension of a
launch holds.  What is looked at is exact: the values are ones, zeros and powers of two."""
import numpy as np
import pytest
import torch

import paper_2508_18182_amd as A
from oracle import layer_oracle as lo

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = A.Context(0)
    yield c
    c.close()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("d", [2**31 - 1, 2**31 - 4, 2**31 - 8])
def test_dropout_of_a_row_of_nearly_2_31_columns(ctx, d):
    """The last columns of such a row: their number plus 8 passes 31 bits.  Nothing behind the row is touched."""
    p, seed, tail = 0.5, 5, 37
    buf = torch.ones(d + 64, dtype=torch.bfloat16, device=DEV)
    buf[d:] = 7.0
    row = buf[:d].view(1, d)
    A.adloco_dropout(ctx, row, row, p, seed)
    assert bool((buf[d:] == 7).all())
    first = (d - tail) // 8 * 8                        # the oracle's mask of the last groups of eight
    col = np.arange(first // 8, (d + 7) // 8, dtype=np.uint64)
    zero = np.zeros_like(col)
    words = lo.philox((col, zero, zero, zero), (seed, 0))
    number = np.stack([(w >> np.uint64(s)) & np.uint64(0xFFFF) for w in words for s in (0, 16)], axis=-1).reshape(-1)[:d - first]
    want = np.where(number >= lo.dropout_threshold(p), 2.0, 0.0)
    assert np.array_equal(buf[first:d].float().cpu().numpy(), want)


# ---- more work items than one dimension of a launch holds: 2^32 -----------------------------------

def test_dropout_of_2_32_rows(ctx):
    rows, seed = 2**32 + 77, 2**40 + 3
    x = torch.ones(rows, 1, dtype=torch.bfloat16, device=DEV)
    A.adloco_dropout(ctx, x, x, 0.5, seed)
    for first in (0, 2**31 - 5, 2**32 - 70, rows - 70):
        want = np.where(lo.dropout_keep(70, 1, 0.5, seed, first), 2.0, 0.0)
        assert np.array_equal(x[first:first + 70].float().cpu().numpy(), want), first
    kept = int((x != 0).sum())                         # (a part that was left out would be all ones)
    assert abs(kept - rows / 2) < 6 * (rows / 4)**0.5 and bool((x[::7] != 1).all())


def test_norm_of_2_28_rows_and_more(ctx):
    rows = 2**28 + 2**20 + 3
    x = torch.full((rows, 1), 4.0, dtype=torch.bfloat16, device=DEV)
    x[::3] = -0.25
    want = x.sign()
    A.adloco_rms_norm(ctx, x, None, 2.0**-100, y=x)
    assert torch.equal(x, want)


@pytest.mark.parametrize("B,d", [(2**26 + 5, 1), (2**26 + 2**20, 3)])
def test_norm_backward_of_2_26_samples(ctx, B, d):
    h = torch.full((B, d), 2.0, dtype=torch.bfloat16, device=DEV)
    h[1::2] = -4.0
    dy = torch.full((B, d), 0.5, dtype=torch.bfloat16, device=DEV)
    sums = torch.full((B, d), 9.0, device=DEV)
    A.adloco_rms_norm_backward(ctx, h, None, dy, 2.0**-100, h, gain_sums=sums)
    sums[1::2] *= -1
    assert float((sums - 0.5).abs().max()) <= 8 * 2.0**-24                      # n = 1 or -1, four roundings
    assert float(h.float().abs().max()) <= 16 * 2.0**-24                        # a constant row: w - n mean(w n) = 0


def test_pack_of_2_23_tiles_and_more(ctx):
    rows = 2**30 + 2**18 + 5
    x = torch.zeros(rows, 1, dtype=torch.bfloat16, device=DEV)
    at = torch.tensor([0, 1, 2**29, 2**30 - 1, 2**30, 2**30 + 1, rows - 1], device=DEV)
    x[at] = 448.0
    across = A.Blocks8.empty(1, rows, DEV)
    across.data.fill_(0x55)
    across.exponent.fill_(0x55)
    A.adloco_pack_blocks(ctx, x, None, across)
    got = torch.nonzero(across.data[0]).flatten()
    assert torch.equal(got, at) and bool((across.data[0][at] == 0x7E).all())
    where = torch.nonzero(across.exponent[:, 0] != 1).flatten()
    assert torch.equal(where, torch.unique(at // 128)) and bool((across.exponent[where, 0] == 127).all())


def test_product_of_few_rows_and_2_28_columns(ctx):
    n = 2**28 + 2**17 + 5
    a, b = A.Blocks8.empty(1, 128, DEV), A.Blocks8.empty(n, 128, DEV)
    a.data.fill_(0x38)                                 # ones
    a.exponent.fill_(127)
    b.data.zero_()
    b.exponent.fill_(127)
    at = torch.tensor([0, 17, 2**27, 2**28 - 1, 2**28, 2**28 + 2**16, n - 1], device=DEV)
    b.data[at, 5] = 0x38
    out = torch.full((1, n), 7.0, dtype=torch.bfloat16, device=DEV)
    ctx.set_tuning("product_blocks", 1)
    try:
        A.adloco_block_product(ctx, a, b, out)
    finally:
        ctx.set_tuning("product_blocks", 0)
    assert torch.equal(torch.nonzero(out[0]).flatten(), at) and bool((out[0][at] == 1).all())
