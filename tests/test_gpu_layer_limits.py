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
