"""Attention of up to 8 query heads to a KV head over pages is off by its result's rounding alone."""

import pytest
import torch

from paged_plain import attend64
from paper_2608_08878_gb300 import dc  # noqa: F401
from test_gpu_paged import BF, HF, filled

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("page,kvh,group,d", [(64, 2, 8, 128), (16, 2, 4, 128), (32, 4, 5, 64), (128, 8, 1, 128)])
def test_one_rounding(page, kvh, group, d, dtype):
    """The distance from 64 bits is that of the rounded 64-bit result. What adds to it: weights of 2^-17 (bf16) or 2^-23 (fp16),
    scores and sums in 32 bits, below 1e-5 of the result together; and the roundings of other values than those of 64
    bits, of at least 8192 in all: 4 standard deviations of their mean square are 4%."""
    lens = [2000, 1, 700, 3001, 64, 1500, 999, 4000]
    cache, tables, n, q = filled(lens, page, kvh, group, d, dtype)
    pick = cache.select(q, tables, n, 10)
    assert q.numel() >= 8192
    for selected in (None, pick):
        out = cache.attend(q, tables, n, selected=selected).double()
        o = attend64(q, cache.k[0], cache.v[0], tables, lens, selected=selected)[0]
        least = (o.to(dtype).double() - o).norm()
        assert float((out - o).norm()) <= 1.04 * float(least) + 1e-5 * float(o.norm())
    cache.check()
