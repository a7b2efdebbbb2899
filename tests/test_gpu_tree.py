"""Attention of drafted trees over a cache against 64 bits: trees of any shape with unused nodes, caches from
empty to evicted ones, rows of different lengths, and what a node does not see."""

import math

import pytest
import torch

from attention64 import attention64, check
from paper_2608_08878_gb300 import dc

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def rand(*shape, seed=0):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(BF)


def tree(batch, T, kind, seed=0):
    g = torch.Generator().manual_seed(seed)
    at = torch.arange(T)
    if kind == "chain":
        p = (at - 1).expand(batch, T)
    elif kind == "flat":
        p = torch.full((batch, T), -1)
    else:
        p = torch.minimum((torch.rand((batch, T), generator=g) * (at + 1)).long() - 1, at - 1)
        if kind == "holes":
            p = torch.where(torch.rand((batch, T), generator=g) < 0.3, torch.randint(-5, 200, (batch, T), generator=g), p)
        if kind == "unused":
            p = torch.full((batch, T), -7)
    return p.to(torch.int32).contiguous().cuda()


def masks(parents):
    """[batch][T][T] truth values on the GPU, walked up node by node."""
    out = torch.zeros(tuple(parents.shape) + (parents.shape[1],), dtype=torch.bool)
    for s, row in enumerate(parents.tolist()):
        for i, p in enumerate(row):
            if p == -1:
                out[s, i, i] = True
            elif 0 <= p < i and bool(out[s, p].any()):
                out[s, i] = out[s, p]
                out[s, i, i] = True
    return out.cuda()


def make(layers, batch, kvh, group, d, n, T, kind="random", seed=0, **kw):
    cache = dc.DistillCache(layers, kvh, d, max(n, 1) + 40, max(1, n - 1), batch=batch, q_heads=kvh * group, **kw)
    k, v = rand(layers, batch, kvh, n, d, seed=seed), rand(layers, batch, kvh, n, d, seed=seed + 1)
    if n:
        cache.append(k, v)
    draft = (rand(layers, batch, T, kvh * group, d, seed=seed + 2), rand(layers, batch, kvh, T, d, seed=seed + 3),
             rand(layers, batch, kvh, T, d, seed=seed + 4), tree(batch, T, kind, seed))
    return cache, draft


def compare(cache, draft, out):
    q, kd, vd, parents = draft
    L, b, T, hq, d = q.shape
    kvh, G = cache.kv_heads, hq // cache.kv_heads
    K, V, lens = cache.buffer(dc.BUF_K), cache.buffer(dc.BUF_V), cache.row_lengths()
    anc = masks(parents)
    for r in range(L * b * kvh):
        lb, g = r // kvh, r % kvh
        layer, s = lb // b, lb % b
        n = int(lens[r])
        used = anc[s].any(-1, keepdim=True)
        seen = torch.cat([used.expand(T, n), anc[s]], 1).repeat_interleave(G, 0)
        qq = q[layer, s, :, g * G: (g + 1) * G].reshape(T * G, d)
        o, _, tol, _ = attention64(qq, torch.cat([K[r, :n], kd[layer, s, g]]), torch.cat([V[r, :n], vd[layer, s, g]]), seen,
                                   d ** -0.5)
        check(out[layer, s, :, g * G: (g + 1) * G].reshape(T * G, d), o, tol, f"row {r} of {n} tokens")


def run(*shape, **kw):
    cache, draft = make(*shape, **kw)
    out = cache.tree_attend(*draft)
    cache.sync()
    assert out.dtype == BF and out.shape == draft[0].shape
    compare(cache, draft, out)


@pytest.mark.parametrize("n", [0, 1, 2, 63, 127, 128, 129, 255, 257, 1000, 4097])
@pytest.mark.parametrize("T", [1, 5, 32])
def test_cache_lengths(n, T):
    run(1, 2, 2, 4, 128, n, T)


@pytest.mark.parametrize("T", [1, 2, 3, 8, 15, 16, 17, 31, 33, 64, 100, 127, 128])
@pytest.mark.parametrize("group", [1, 2, 4, 8])
def test_tree_sizes(T, group):
    run(1, 1, 2, group, 64, 300, T)


@pytest.mark.parametrize("kind", ["random", "chain", "flat", "holes", "unused"])
@pytest.mark.parametrize("d", [64, 128])
def test_tree_shapes(kind, d):
    run(2, 3, 2, 4, d, 500, 40, kind=kind)
    run(1, 2, 1, 8, d, 77, 128, kind=kind)


def test_many_rows_and_long_rows():
    run(4, 4, 8, 4, 128, 700, 16)
    run(1, 1, 2, 4, 128, 30000, 9)
    run(1, 1, 1, 1, 64, 70001, 1)


def test_nothing_drafted():
    cache, draft = make(1, 1, 2, 2, 64, 10, 0)
    assert cache.tree_attend(*draft).shape == (1, 1, 0, 4, 64)


def test_over_an_evicted_cache_and_rows_of_different_lengths():
    cache, draft = make(2, 1, 2, 4, 128, 600, 12)
    cache.step(rand(2, 1, 8, 128, seed=8), rand(2, 1, 2, 128, seed=9), rand(2, 1, 2, 128, seed=10), budget=200)
    compare(cache, draft, cache.tree_attend(*draft))
    cache.set_row_budgets([180, 7, 130, 1])
    cache.step(rand(2, 1, 8, 128, seed=11), rand(2, 1, 2, 128, seed=12), rand(2, 1, 2, 128, seed=13))
    assert list(cache.row_lengths()) == [180, 7, 130, 1]
    before = [cache.buffer(w).clone() for w in (dc.BUF_K, dc.BUF_V, dc.BUF_POS, dc.BUF_S)]
    compare(cache, draft, cache.tree_attend(*draft))
    # the cache is as it was
    assert all(torch.equal(a.view(torch.uint8), cache.buffer(w).view(torch.uint8))
               for a, w in zip(before, (dc.BUF_K, dc.BUF_V, dc.BUF_POS, dc.BUF_S)))
    cache.sync()


def test_one_node_is_the_decode_step():
    cache, (q, kd, vd, parents) = make(2, 2, 2, 4, 128, 400, 1, kind="chain")
    out = cache.tree_attend(q, kd, vd, parents)
    ref = cache.decode_step(q[:, :, 0], kd[:, :, :, 0], vd[:, :, :, 0])
    assert float((out[:, :, 0].float() - ref).abs().max()) <= 2.0 ** -8 * float(vd.abs().max())


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_what_a_node_does_not_see_leaves_it_alone(bad):
    """Drafted tokens off a node's path, and the slots past a row's tokens (evicted ones), hold NaN or infinities."""
    k, v = rand(1, 2, 2, 3, 64, seed=20), rand(1, 2, 2, 3, 64, seed=21)
    v[:] = bad
    cache, (q, kd, vd, parents) = make(1, 2, 2, 2, 64, 90, 20, scorer=2, n_sinks=90)
    cache.append(k, v)
    cache.decode_step(rand(1, 2, 4, 64, seed=22), rand(1, 2, 2, 64, seed=23), rand(1, 2, 2, 64, seed=24))
    cache.evict(90)  # the sinks stay, the tokens with the bad values go
    vd[0, 0, 1, 6] = bad
    kd[0, 1, 0, 9] = bad
    out = cache.tree_attend(q, kd, vd, parents)
    cache.sync()
    anc = masks(parents)
    sees = torch.zeros((2, 20, 4), dtype=torch.bool, device="cuda")
    sees[0, :, 2:] |= anc[0, :, 6, None]
    sees[1, :, :2] |= anc[1, :, 9, None]
    assert bool(torch.isfinite(out[0][~sees]).all())
    assert not bool(torch.isfinite(out[0][sees]).all(-1).any())
    clean_v, clean_k = vd.clone(), kd.clone()
    clean_v[0, 0, 1, 6], clean_k[0, 1, 0, 9] = 0, 0
    ref = cache.tree_attend(q, clean_k, clean_v, parents)
    compare(cache, (q, clean_k, clean_v, parents), ref)
    keep = ~sees
    # (a row whose tile holds a value that is not finite may be summed in another order)
    assert float((out[0][keep].float() - ref[0][keep].float()).abs().max()) <= 2.0 ** -7 * float(clean_v.abs().max())


def test_refusals():
    cache, (q, kd, vd, parents) = make(1, 2, 2, 2, 64, 30, 4)
    bad = {
        "parents of another batch": (q, kd, vd, parents[:1].contiguous()),
        "parents of another type": (q, kd, vd, parents.long()),
        "parents on the host": (q, kd, vd, parents.cpu()),
        "q one node short": (q[:, :, :3].contiguous(), kd, vd, parents),
        "q of another type": (q.half(), kd, vd, parents),
        "k_draft not dense": (q, kd.transpose(3, 4), vd, parents),
        "too many nodes": (rand(1, 2, 129, 4, 64), rand(1, 2, 2, 129, 64), rand(1, 2, 2, 129, 64), tree(2, 129, "chain")),
    }
    for what, args in bad.items():
        with pytest.raises(dc.DCError) as e:
            cache.tree_attend(*args)
        assert e.value.status == dc.DC_ERR_INVALID_ARG, what
    compare(cache, (q, kd, vd, parents), cache.tree_attend(q, kd, vd, parents))


def test_a_captured_call_replays():
    """A row in parts: the first call makes the buffer for them, so it is refused in a capture; a later one is captured
    and replays on what its tensors then hold."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        cache, (q, kd, vd, parents) = make(1, 1, 2, 4, 64, 5000, 4)
        out = torch.zeros_like(q)
        cache.sync()
        refused = torch.cuda.CUDAGraph()
        with torch.cuda.graph(refused, stream=stream):
            out.add_(0)
            with pytest.raises(dc.DCError) as e:
                cache.tree_attend(q, kd, vd, parents, out)
        assert e.value.status == dc.DC_ERR_STATE
        cache.tree_attend(q, kd, vd, parents, out)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            cache.tree_attend(q, kd, vd, parents, out)
        q.copy_(rand(1, 1, 4, 8, 64, seed=77))
        graph.replay()
        stream.synchronize()
        compare(cache, (q, kd, vd, parents), out)


def test_an_allocation_failure_leaves_the_cache_usable():
    cache, draft = make(1, 1, 2, 4, 64, 5000, 4)
    try:
        dc.debug_fail_alloc(0)
        with pytest.raises(dc.DCError) as e:
            cache.tree_attend(*draft)
        assert e.value.status == dc.DC_ERR_OOM
    finally:
        dc.debug_fail_alloc(-1)
    compare(cache, draft, cache.tree_attend(*draft))
    cache.sync()


def test_graph_mode_refuses():
    cache, draft = make(1, 1, 2, 4, 64, 130, 3, window=2)
    for i in range(3):
        cache.step(rand(1, 1, 8, 64, seed=30 + i), rand(1, 1, 2, 64, seed=40 + i), rand(1, 1, 2, 64, seed=50 + i))
    cache.set_graph_mode(True)
    with pytest.raises(dc.DCError) as e:
        cache.tree_attend(*draft)
    assert e.value.status == dc.DC_ERR_STATE
    cache.set_graph_mode(False)
    compare(cache, draft, cache.tree_attend(*draft))


def test_row_offsets_past_32_bits():
    """The last row's keys lie past 2^32 bytes into the cache's."""
    n, d = 2_300_000, 128
    cache = dc.DistillCache(1, 8, d, n + 8, n - 1, q_heads=8, window=1)
    k, v = (torch.empty((1, 1, 8, n, d), dtype=BF, device="cuda").normal_() for _ in range(2))
    cache.append(k, v)
    q, kd, vd = rand(1, 1, 3, 8, d), rand(1, 1, 8, 3, d, seed=1), rand(1, 1, 8, 3, d, seed=2)
    out = cache.tree_attend(q, kd, vd, tree(1, 3, "chain"))
    cache.sync()
    seen = torch.ones((3, n + 3), dtype=torch.bool, device="cuda")
    seen[:, n:] = torch.tril(torch.ones((3, 3), device="cuda")).bool()
    for g in (0, 7):
        o, _, tol, _ = attention64(q[0, 0, :, g], torch.cat([k[0, 0, g], kd[0, 0, g]]), torch.cat([v[0, 0, g], vd[0, 0, g]]),
                                   seen, d ** -0.5)
        check(out[0, 0, :, g], o, tol)


@pytest.mark.parametrize("layers,batch,kvh,group,d,n,T", [
    (10, 4, 4, 8, 64, 515, 64), (7, 3, 4, 8, 128, 300, 96), (5, 4, 8, 8, 64, 129, 128), (19, 1, 8, 4, 128, 900, 100),
    (1, 1, 8, 8, 128, 5000, 70), (38, 2, 1, 8, 64, 1100, 33)])
def test_several_pairs_of_query_tiles(layers, batch, kvh, group, d, n, T):
    run(layers, batch, kvh, group, d, n, T)


def test_random_shapes():
    import random
    r = random.Random(5)
    for i in range(30):
        group = r.choice([1, 2, 4, 8])
        run(r.choice([1, 2, 5]), r.choice([1, 3, 8]), r.choice([1, 2, 8]), group, r.choice([64, 128]), int(2 ** r.uniform(0, 11)),
            min(128, int(2 ** r.uniform(0, 7.2))), kind=r.choice(["random", "chain", "flat", "holes"]), seed=i)


@pytest.mark.parametrize("layers,batch,kvh,group,d,n,T,kind", [
    (5, 4, 8, 4, 128, 410, 8, "random"), (3, 7, 8, 4, 64, 1000, 32, "holes"), (1, 153, 1, 8, 64, 130, 16, "random"),
    (9, 39, 1, 2, 128, 1, 5, "chain"), (40, 2, 4, 1, 128, 511, 100, "random"), (2, 50, 2, 4, 64, 0, 3, "flat"),
    (32, 8, 2, 4, 128, 513, 1, "chain"), (1, 155, 2, 4, 128, 300, 7, "unused")])
def test_many_short_rows(layers, batch, kvh, group, d, n, T, kind):
    run(layers, batch, kvh, group, d, n, T, kind=kind)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_what_a_node_does_not_see_in_many_short_rows(bad):
    for d, rows in ((64, (3, 53, 1)), (128, (5, 8, 4))):
        cache, (q, kd, vd, parents) = make(*rows, 4, d, 200, 20)
        ref = cache.tree_attend(q, kd, vd, parents)
        compare(cache, (q, kd, vd, parents), ref)
        kd[:, :, :, 19], vd[:, :, :, 19] = bad, bad  # (no node follows the last one)
        out = cache.tree_attend(q, kd, vd, parents)
        cache.sync()
        assert float((out[:, :, :19].float() - ref[:, :, :19].float()).abs().max()) <= 2.0 ** -7 * float(vd[:, :, :, :19].abs().max())
        assert not bool(torch.isfinite(out[:, :, 19].float()).all(-1).any())


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("rows,group,d,n,T", [
    ((1, 2, 2), 4, 128, 300, 6), ((1, 2, 2), 8, 64, 300, 100), ((1, 3, 1), 1, 128, 0, 9),  # one item a row or two
    ((3, 53, 1), 4, 64, 200, 6),                                                           # two rows an item
    ((1, 1, 2), 4, 128, 5000, 6), ((1, 1, 1), 8, 64, 3000, 70)])                           # rows in parts
def test_queries_of_unused_nodes_may_hold_anything(rows, group, d, n, T, bad):
    """An unused node's output is 0 and no other node's changes, whatever its query holds."""
    cache, (q, kd, vd, parents) = make(*rows, group, d, n, T, kind="chain")
    parents[:, T // 2] = -7     # (and so is all of the chain behind it)
    parents[:, T // 2 + 1] = 0  # but for this node and what follows it
    want = cache.tree_attend(q, kd, vd, parents)
    compare(cache, (q, kd, vd, parents), want)
    q[:, :, T // 2] = bad
    out = cache.tree_attend(q, kd, vd, parents)
    cache.sync()
    assert bool((out[:, :, T // 2] == 0).all())
    assert torch.equal(out.view(torch.int16), want.view(torch.int16))


def test_drafts_and_queries_the_other_way_round_are_refused():
    """[nodes][heads] where [heads][nodes] is meant, and the reverse, dense: as many elements, another order."""
    cache, (q, kd, vd, parents) = make(1, 3, 2, 2, 64, 30, 4)
    swap = lambda t: t.transpose(2, 3).contiguous()  # noqa: E731
    want = cache.tree_attend(q, kd, vd, parents)
    q5, k5, v5, p5 = rand(1, 3, 5, 4, 64), rand(1, 3, 2, 5, 64, seed=1), rand(1, 3, 2, 5, 64, seed=2), tree(3, 5, "chain")
    bad = {"k_draft": (q, swap(kd), vd, parents), "v_draft": (q, kd, swap(vd), parents), "q": (swap(q5), k5, v5, p5),
           "out": (q5, k5, v5, p5, torch.empty_like(swap(q5)))}
    for what, args in bad.items():
        with pytest.raises(dc.DCError) as e:
            cache.tree_attend(*args)
        assert e.value.status == dc.DC_ERR_INVALID_ARG and what in str(e.value)
    # views in the same order are as good
    for qv, kv in ((q[0], kd[0]), (q.view(3, 4, 2, 2, 64), kd.view(6, 4, 64)), (q.view(1, 3, 4, 256), kd.view(-1)),
                   (q.view(1, 3, 4, 2, 2, 64), kd)):
        assert torch.equal(cache.tree_attend(qv, kv, vd, parents).view(-1), want.view(-1))


def test_inputs_of_another_stream_are_kept_until_they_are_read():
    """The cache on a stream of its own that is busy; the caller drops the inputs, and the default stream's next tensors
    would take their places."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        cache, kept = make(1, 2, 2, 4, 64, 300, 6)
    for busy in (False, True):  # (first launches load kernels, and wait)
        torch.cuda.synchronize()
        draft = [t.clone() for t in kept]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            if busy:
                torch.cuda._sleep(1 << 28)
            done = torch.cuda.Event()
        out = cache.tree_attend(*draft)
        done.record(side)
        shapes = [(t.shape, t.dtype) for t in draft]
        draft.clear()
        over = [torch.full(s, 1, dtype=d, device="cuda") for s, d in shapes]
        torch.cuda.current_stream().synchronize()
        assert not busy or not done.query()
        torch.cuda.synchronize()
        compare(cache, kept, out)
        del over
