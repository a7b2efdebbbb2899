"""Attention over shared prefixes reads what kernels directly before it have written in place: its own tokens' kernel
starts beside the prefixes' one."""

import pytest
import torch

from paper_2608_08878_gb300 import dc

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("d,page,group", [(128, 64, 4), (64, 16, 8)])
def test_inputs_that_change_in_place_directly_before(d, page, group):
    """A step of appends, lengths, tables and queries written in place in front of each call, captured and replayed many times
    with nothing between the steps; the same calls one by one with everything waited for give the same bits."""
    kvh, S, shared_tokens, width, steps = 2, 24, 4 * page, 16, 40
    g = torch.Generator(device="cuda").manual_seed(11)
    T0 = torch.cat([torch.arange(4, device="cuda").expand(S, 4), 4 + torch.arange(S * (width - 4), device="cuda").view(S, -1)], 1).int()
    start = torch.randint(shared_tokens, shared_tokens + 3 * page, (S,), device="cuda", generator=g).int()
    # of each step: which of two homes its own pages have, how many tokens that are there already it takes up, its query and tokens
    move = torch.randint(0, 2, (steps, S, 1), device="cuda", generator=g).int() * (S * (width - 4))
    by = torch.randint(0, 3, (steps, S), device="cuda", generator=g).int()
    x = torch.randn((steps, S, kvh * (group + 2), d), device="cuda", generator=g).to(BF)
    f = torch.rand(d // 2, device="cuda", generator=g)
    cache = dc.PagedCache(1, 4 + 2 * S * width, kvh, d, page_size=page, q_heads=kvh * group)
    shared = cache.share([S - 1], [shared_tokens])  # (the last sequence reads those pages by itself)
    first = [torch.randn(t.shape, device="cuda", generator=g).to(BF) for t in cache._memory]
    tables, lens, at = T0.clone(), start.clone(), torch.zeros((), dtype=torch.long, device="cuda")
    outs = torch.empty((steps, S, kvh * group, d), dtype=BF, device="cuda")
    lses = torch.empty((steps, S, kvh * group), device="cuda")

    def step():
        y = x.index_select(0, at.view(1))[0]
        tables[:, 4:] = T0[:, 4:] + move.index_select(0, at.view(1))[0]
        lens.add_(by.index_select(0, at.view(1))[0])
        q = cache.append(y[:, : kvh * group], y[:, kvh * group: kvh * (group + 1)], y[:, kvh * (group + 1):], tables, lens, f)
        lens.add_(1)
        o, z = cache.attend(q, tables, lens, shared=shared, with_lse=True)
        outs.index_copy_(0, at.view(1), o[None])
        lses.index_copy_(0, at.view(1), z[None])
        at.add_(1)

    def begin():
        for t, v in zip(cache._memory, first):
            t.copy_(v)
        tables.copy_(T0)
        lens.copy_(start)
        at.zero_()
        outs.zero_()

    begin()
    for _ in range(steps):
        step()
        torch.cuda.synchronize()
    cache.check()
    want, want_z = outs.clone(), lses.clone()
    graph = torch.cuda.CUDAGraph()
    begin()
    with torch.cuda.graph(graph):
        step()
    for _ in range(10):
        begin()
        for _ in range(steps):
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs, want) and torch.equal(lses, want_z)
        begin()
        for _ in range(steps):
            step()
        torch.cuda.synchronize()
        assert torch.equal(outs, want) and torch.equal(lses, want_z)
    cache.check()
