"""Attention of up to 8 query heads to a KV head over pages is off by its result's rounding alone."""

import math

import pytest
import torch

from attention64 import check
from paged_plain import attend64
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


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("scale", [None, 0.4, 1e-6])
@pytest.mark.parametrize("group", [1, 4, 8, 12])
def test_infinite_values(group, scale, dtype):
    """Whatever weight of a token, down to 2^-30 of the largest, meets an infinite value: the result is infinite."""
    lens = [1, 2, 130, 700, 64, 3000]
    cache, tables, n, q = filled(lens, 32, 2, group, 64, dtype)
    clean = cache.attend(q, tables, n, scale=scale)
    at = []
    for s, m in enumerate(lens):
        for j, t in enumerate({0, m // 2, m - 1}):  # in a dim of each token's own
            cache.v[0][int(tables[s, t // 32]), :, t % 32, 10 + j] = math.inf if j % 2 == 0 else -math.inf
            at.append((s, t, 10 + j))
        p = tables[s, : -(-m // 32)].long()  # the token of each KV head's first query head that weighs most
        k = cache.k[0][p].transpose(0, 1).flatten(1, 2)[:, :m]
        for h in range(2):
            t = int((k[h].float() @ q[s, h * group].float()).argmax())
            cache.v[0][int(tables[s, t // 32]), h, t % 32, 3] = math.inf
    out = cache.attend(q, tables, n, scale=scale)
    cache.check()
    o, _, tol, _ = attend64(q, cache.k[0], cache.v[0], tables, lens, scale)
    weighs = torch.ones_like(o, dtype=torch.bool)
    for s, t, dim in at:
        p = tables[s, : -(-lens[s] // 32)].long()
        k = cache.k[0][p].transpose(0, 1).flatten(1, 2)[:, : lens[s]].double()
        z = (q[s].double().view(2, group, 64) @ k.transpose(1, 2)) * (64 ** -0.5 if scale is None else scale)
        weighs[s, :, dim] = ((z[..., t] - z.amax(-1)) > -30 * math.log(2)).flatten()
    assert int(weighs.sum()) > 0.9 * weighs.numel()
    check(torch.where(weighs, out.double(), 0.0), torch.where(weighs, o, 0.0), tol)
    assert torch.equal(out[..., 20:], clean[..., 20:]) and torch.equal(out[..., :3], clean[..., :3])
