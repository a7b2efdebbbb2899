"""Shared prefixes: values that are not finite in shared tokens, page numbers outside the pool one at a time, and as many query
heads to a KV head as there may be."""

import math

import pytest
import torch

from attention64 import check
from paged_plain import attend64
from paper_2608_08878_gb300 import dc
from test_gpu_paged import BF, HF, NAN, filled, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [96, 160, 256, 640])
@pytest.mark.parametrize("size,group,d,dtype", [(1, 4, 128, BF), (3, 4, 128, BF), (40, 4, 128, BF), (70, 4, 64, HF), (9, 16, 64, BF),
                                                (3, 33, 128, HF)])
def test_shared_values_that_are_not_finite(tokens, size, group, d, dtype):
    """In a full key tile of 128 tokens and in one that the prefix fills in part, behind one tile of query rows and behind two:
    who sees such a value has it in its result, in that head and dim alone."""
    page, kvh = 32, 3
    common = [(0, size, tokens), (size, 2, 64)]
    lens = [tokens + (i * 23) % 70 for i in range(size)] + [64, 90, 30]
    cache, tables, n, q = filled(lens, page, kvh, group, d, dtype, common=common)
    at = lambda s, t: (int(tables[s, t // page]), t % page)  # noqa: E731
    shared = cache.share([size, 2], [tokens, 64])
    clean = cache.attend(q, tables, n, shared=shared)
    p, i = at(0, tokens - 1)  # (the last tile's last token)
    cache.v[0][p, 0, i, 5] = math.inf
    p, i = at(0, tokens // 2)
    cache.v[0][p, 0, i, 6] = -math.inf
    cache.v[0][p, 0, i, 7] = NAN
    p, i = at(0, tokens - 30)
    cache.k[0][p, 1, i, 9] = NAN
    p, i = at(size, 40)
    cache.k[0][p, 2, i, 1] = NAN
    out, lse = cache.attend(q, tables, n, shared=shared, with_lse=True)
    cache.check()
    o, z, tol, tolz = attend64(q, cache.k[0], cache.v[0], tables, lens, shared=common)
    check(out, o, tol, "out")
    check(lse, z, tolz, "lse")
    x, c = out.view(-1, kvh, group, d), clean.view(-1, kvh, group, d)
    assert bool((x[:size, 0, :, 5] == math.inf).all()) and bool((x[:size, 0, :, 6] == -math.inf).all())
    assert bool(torch.isnan(x[:size, 1]).all()) and bool(torch.isnan(x[size: size + 2, 2]).all())
    # everything else has the bits of before
    assert torch.equal(x[:size, 0, :, :5], c[:size, 0, :, :5]) and torch.equal(x[:size, 0, :, 8:], c[:size, 0, :, 8:])
    assert torch.equal(x[:size, 2], c[:size, 2]) and torch.equal(x[size:, :2], c[size:, :2]) and torch.equal(x[size + 2:], c[size + 2:])


@pytest.mark.parametrize("bad", [-1, "pool", 2 ** 31 - 1, -2 ** 31])
@pytest.mark.parametrize("where", ["shared", "own"])
def test_each_page_number_outside_the_pool_is_reported(bad, where):
    lens, common = [300, 200, 130], [(0, 2, 128)]
    cache, tables, n, q = filled(lens, 32, 2, 4, 64, common=common)
    shared = cache.share([2], [128])
    cache.attend(q, tables, n, shared=shared)
    cache.check()
    tables[(0, 1) if where == "shared" else (2, 3)] = cache.pages if bad == "pool" else bad
    cache.attend(q, tables, n, shared=shared)
    with pytest.raises(dc.DCError) as e:
        cache.check()
    assert e.value.status == dc.DC_ERR_DEVICE and "page" in str(e.value)


@pytest.mark.parametrize("group", [16, 17, 48, 64, 65, 100, 128])
@pytest.mark.parametrize("size,d,dtype", [(1, 64, BF), (3, 128, HF), (12, 128, BF)])
def test_shared_by_many_query_heads(group, size, d, dtype):
    run([640 + (i * 13) % 70 for i in range(size)] + [50], 64, 2, group, d, dtype, common=[(0, size, 640)])
    run([96 + (i * 13) % 70 for i in range(size)] + [0], 16, 1, group, d, dtype, common=[(0, size, 96)])
