"""Attention of packed prompts against 64 bits: lengths from none to long ones, groups, types, layouts,
rows that see nothing, values that are not finite in places that a row does not see."""

import math

import pytest
import torch

from attention64 import attention64, check
from paper_2608_08878_gb300 import dc

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def inputs(q_lens, k_lens, kvh, group, d, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randn((sum(q_lens), kvh * group, d), device="cuda", generator=g).to(dtype)
    k = torch.randn((sum(k_lens), kvh, d), device="cuda", generator=g).to(dtype)
    v = torch.randn((sum(k_lens), kvh, d), device="cuda", generator=g).to(dtype)
    return q, k, v


def seen_by(t, ql, kl, causal):
    at = torch.arange(kl, device="cuda")
    return (at <= t[:, None] + (kl - ql)) if causal else (at < kl).expand(len(t), kl)


def compare(out, lse, q, k, v, q_lens, k_lens, causal=True, scale=None, rows=512):
    """Every row of short sequences; of longer ones the first and last `rows` / 2 and as many in between."""
    kvh, group, d = k.shape[1], q.shape[1] // k.shape[1], q.shape[2]
    scale = d ** -0.5 if scale is None else scale
    q0 = k0 = 0
    for s, (ql, kl) in enumerate(zip(q_lens, k_lens)):
        t = torch.arange(ql, device="cuda")
        if ql > rows:
            mid = torch.randint(0, ql, (rows // 2,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(s))
            t = torch.unique(torch.cat([t[: rows // 4], t[-rows // 4:], mid]))
        step = max(1, (1 << 26) // max(1, kvh * group * kl))
        for part in t.split(step):
            if not len(part):
                continue
            qq = q[q0 + part].view(len(part), kvh, group, d).permute(1, 2, 0, 3)
            kk, vv = (x[k0: k0 + kl].transpose(0, 1)[:, None] for x in (k, v))
            o, z, tol, tolz = attention64(qq, kk, vv, seen_by(part, ql, kl, causal), scale)
            what = f"sequence {s} ({ql}, {kl})"
            check(out[q0 + part].view(len(part), kvh, group, d).permute(1, 2, 0, 3), o, tol, what)
            if lse is not None:
                check(lse[q0 + part].view(len(part), kvh, group).permute(1, 2, 0), z, tolz, what + " lse")
        q0, k0 = q0 + ql, k0 + kl


def run(q_lens, kvh, group, d, dtype=BF, k_lens=None, causal=True, seed=0):
    k_lens = k_lens or q_lens
    q, k, v = inputs(q_lens, k_lens, kvh, group, d, dtype, seed)
    plan = dc.PromptPlan(q_lens, kvh, d, q_heads=kvh * group, k_lens=k_lens, causal=causal)
    out, lse = plan.attend(q, k, v, with_lse=True)
    plan.check()
    assert out.dtype == dtype and lse.dtype == torch.float32
    compare(out, lse, q, k, v, q_lens, k_lens, causal)


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 1000])
@pytest.mark.parametrize("group", [1, 4])
def test_one_prompt_of_any_length(n, group):
    run([n], 2, group, 128)


@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 6, 7, 8, 12, 16, 33, 64, 65, 128])
@pytest.mark.parametrize("d", [64, 128])
def test_groups(group, d):
    run([37, 1, 150], 2, group, d)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_packed_sequences(dtype, d, causal):
    run([1, 17, 0, 130, 64, 301, 777, 2], 4, 4, d, dtype, causal=causal)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("causal", [True, False])
def test_chunks_and_turns_after_long_contexts(dtype, causal):
    run([100, 1, 33, 512, 7], 2, 4, 128, dtype, k_lens=[1100, 5000, 33, 700, 129], causal=causal)


def test_single_tokens_over_long_caches():
    run([1] * 6, 8, 4, 128, k_lens=[20000, 1, 127, 128, 129, 4097])
    run([1], 1, 8, 64, k_lens=[50001])
    run([2, 1], 1, 1, 128, k_lens=[33333, 3])


def test_long_prompts():
    run([8192], 2, 4, 128)
    run([4099, 4097], 1, 8, 64)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_rows_that_see_nothing(dtype):
    # more queries than keys: the first ones see none; sequences with no key at all, and all of them so
    run([10, 5, 300, 64], 2, 4, 128, dtype, k_lens=[4, 0, 130, 64])
    run([3, 70], 2, 2, 64, dtype, k_lens=[0, 0])
    run([3, 70], 2, 2, 64, dtype, k_lens=[0, 0], causal=False)


def test_nothing_to_do():
    plan = dc.PromptPlan([0, 0], 2, 64, q_heads=4, k_lens=[0, 5])
    q, k, v = inputs([0], [5], 2, 2, 64, BF)
    assert plan.attend(q, k, v).shape == (0, 4, 64)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("d", [64, 128])
def test_what_a_row_does_not_see_leaves_it_alone(bad, d):
    """Later tokens of the prompt, and the next sequence's, hold NaN or infinities in keys and values; the rows
    that see an infinite or NaN value have it."""
    lens = [200, 1, 77, 300]
    q, k, v = inputs(lens, lens, 2, 4, d, BF)
    v[150, 0, 3] = bad   # seen by rows 150.. of sequence 0
    v[201:278] = bad     # all of sequence 2
    k[270, 1] = math.nan
    v[278 + 299, 1] = bad  # the last token
    plan = dc.PromptPlan(lens, 2, d, q_heads=8)
    out, lse = plan.attend(q, k, v, with_lse=True)
    # the rows that see the NaN key are NaN
    assert bool(torch.isnan(out[270:278, 4:]).all()) and bool(torch.isnan(lse[270:278, 4:]).all())
    k2 = k.clone()
    k2[270, 1] = 0
    keep = torch.ones(out.shape[:2], dtype=torch.bool, device="cuda")
    keep[270:278, 4:] = False
    o2, l2 = plan.attend(q, k2, v, with_lse=True)
    assert torch.equal(out[keep].view(torch.int16), o2[keep].view(torch.int16)) and torch.equal(lse[keep], l2[keep])
    compare(o2, l2, q, k2, v, lens, lens)


def test_keys_of_minus_infinity_have_no_weight():
    """A score of -infinity has no weight; a row of nothing else is 0 / 0."""
    q, k, v = inputs([40], [40], 1, 1, 64, BF)
    q[..., 0], k[..., 0] = 1.0, 0.0
    k[5, 0, 0] = -math.inf
    out, lse = dc.PromptPlan([40], 1, 64, q_heads=1).attend(q, k, v, with_lse=True)
    keep = torch.arange(40, device="cuda") != 5
    seen = seen_by(torch.arange(40, device="cuda"), 40, 40, True)[:, keep]
    o, z, tol, tolz = attention64(q[:, 0], k[keep, 0], v[keep, 0], seen, 0.125)
    check(out[:, 0], o, tol)
    check(lse[:, 0], z, tolz)
    k[0, 0, 0] = -math.inf
    out = dc.PromptPlan([40], 1, 64, q_heads=1).attend(q, k, v)
    assert bool(torch.isnan(out[0]).all()) and bool(torch.isfinite(out[1:]).all())


def test_large_scores_and_scales():
    q, k, v = inputs([260], [260], 2, 2, 128, BF)
    for f, scale in ((8.0, None), (1.0, 3.0), (1.0, 1e-4), (30.0, None)):
        qq = (q * f).to(BF)
        out, lse = dc.PromptPlan([260], 2, 128, q_heads=4).attend(qq, k, v, with_lse=True, scale=scale)
        compare(out, lse, qq, k, v, [260], [260], scale=scale)


def test_rising_maxima():
    """Scores that rise along the keys, and fall: every tile brings a new maximum, or none does."""
    for sign in (1, -1):
        q, k, v = inputs([1500], [1500], 1, 4, 64, BF)
        ramp = sign * torch.linspace(-40, 40, 1500, device="cuda")
        q[..., 0], k[:, 0, 0] = 8.0, ramp.to(BF)
        out, lse = dc.PromptPlan([1500], 1, 64, q_heads=4).attend(q, k, v, with_lse=True)
        compare(out, lse, q, k, v, [1500], [1500])


def test_views_of_a_fused_projection_and_head_major_keys():
    lens, kvh, group, d = [70, 200], 2, 4, 128
    q, k, v = inputs(lens, lens, kvh, group, d, BF)
    fused = torch.cat([q, k, v], 1).contiguous()
    plan = dc.PromptPlan(lens, kvh, d, q_heads=kvh * group)
    want = plan.attend(q, k, v)
    qv, kv, vv = fused[:, : kvh * group], fused[:, kvh * group: kvh * group + kvh], fused[:, kvh * group + kvh:]
    assert torch.equal(plan.attend(qv, kv, vv), want)
    kh, vh = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (k, v))
    out = torch.full_like(want, 7.0)
    assert plan.attend(q, kh, vh, out=out).data_ptr() == out.data_ptr() and torch.equal(out, want)
    one = dc.PromptPlan([1, 1], kvh, d, q_heads=kvh * group, k_lens=[70, 200])
    at = [69, 269]
    compare(one.attend(q[at], k, v), None, q[at], k, v, [1, 1], [70, 200])


def test_offsets_past_32_bits():
    """Keys and values 2^25 elements apart: the last of 150 lies past 2^32 elements."""
    step, n, d = 1 << 25, 150, 64
    buf = torch.empty(step * (n - 1) + 2 * d, dtype=BF, device="cuda")
    q, k, v = inputs([n], [n], 1, 2, d, BF)
    kb = buf.as_strided((n, 1, d), (step, d, 1))
    vb = buf.as_strided((n, 1, d), (step, d, 1), d)
    kb.copy_(k)
    vb.copy_(v)
    plan = dc.PromptPlan([n], 1, d, q_heads=2)
    assert torch.equal(plan.attend(q, kb, vb), plan.attend(q, k, v))


def test_same_results_every_time_on_every_stream_and_from_a_graph():
    lens, k_lens = [300, 1, 40], [300, 9000, 2000]
    q, k, v = inputs(lens, k_lens, 2, 4, 128, BF)
    plan = dc.PromptPlan(lens, 2, 128, q_heads=8, k_lens=k_lens)
    want, lse = plan.attend(q, k, v, with_lse=True)
    for _ in range(5):
        o, z = plan.attend(q, k, v, with_lse=True)
        assert torch.equal(o, want) and torch.equal(z, lse)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [plan.attend(q, k, v, stream=s) for s in streams for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    out = torch.zeros_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.attend(q, k, v, out=out)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_refusals():
    q, k, v = inputs([8], [8], 2, 2, 64, BF)
    plan = dc.PromptPlan([8], 2, 64, q_heads=4)
    odd = torch.zeros(8 * 4 * 64 + 1, dtype=BF, device="cuda")[1:].view(8, 4, 64)
    bad = {
        "q of another type": lambda: plan.attend(q.float(), k, v),
        "k of another type": lambda: plan.attend(q, k.half(), v),
        "k on the host": lambda: plan.attend(q, k.cpu(), v),
        "one token short": lambda: plan.attend(q[:7], k, v),
        "v one token short": lambda: plan.attend(q, k, v[:7]),
        "another head count": lambda: plan.attend(q[:, :2], k, v),
        "another head size": lambda: plan.attend(q[..., :32], k[..., :32], v[..., :32]),
        "heads off 16 bytes": lambda: plan.attend(odd, k, v),
        "one key for all tokens": lambda: plan.attend(q, k[:1].expand(8, 2, 64), v),
        "an output of another shape": lambda: plan.attend(q, k, v, out=q[:7]),
        "an output that is not dense": lambda: plan.attend(q, k, v, out=q.transpose(0, 1)),
        "scale 0": lambda: plan.attend(q, k, v, scale=0.0),
        "a scale that is not finite": lambda: plan.attend(q, k, v, scale=math.inf),
    }
    for what, call in bad.items():
        with pytest.raises(dc.DCError) as e:
            call()
        assert e.value.status == dc.DC_ERR_INVALID_ARG, what
    compare(plan.attend(q, k, v), None, q, k, v, [8], [8])
    plan.close()
    with pytest.raises(dc.DCError):
        plan.attend(q, k, v)


def test_the_workspace_is_checked():
    """A plan that divides long key sequences needs its workspace: none, too small and off 16 bytes are refused."""
    import ctypes as C
    q, k, v = inputs([1], [20000], 1, 4, 64, BF)
    plan = dc.PromptPlan([1], 1, 64, q_heads=4, k_lens=[20000])
    assert plan.workspace_bytes > 0
    out, work = torch.empty_like(q), torch.empty(plan.workspace_bytes + 16, dtype=torch.uint8, device="cuda")
    for at, n in ((0, plan.workspace_bytes), (work.data_ptr(), plan.workspace_bytes - 1), (work.data_ptr() + 8, plan.workspace_bytes)):
        a = dc.dc_prompt_args(0, 0.125, q.data_ptr(), k.data_ptr(), v.data_ptr(), 256, 64, 64, 64, 64, 64, out.data_ptr(), 0, at, n)
        assert dc.lib().dc_prompt_attend(plan._p, C.byref(a), None) == dc.DC_ERR_INVALID_ARG


def test_random_shapes():
    import random
    r = random.Random(11)
    for i in range(30):
        count = r.randint(1, 6)
        q_lens = [int(2 ** r.uniform(0, 10)) - r.randint(0, 1) for _ in range(count)]
        k_lens = [max(0, x + r.choice([0, 0, -2, int(2 ** r.uniform(0, 11))])) for x in q_lens]
        run(q_lens, r.choice([1, 2, 3, 8]), r.choice([1, 2, 3, 4, 5, 8]), r.choice([64, 128]), r.choice([BF, HF]), k_lens,
            r.random() < 0.8, seed=i)


def test_lse_off_4_bytes_is_refused():
    import ctypes as C
    q, k, v = inputs([8], [8], 2, 2, 64, BF)
    plan, out, lse = dc.PromptPlan([8], 2, 64, q_heads=4), torch.empty_like(q), torch.empty(64, device="cuda")
    for at, status in ((2, dc.DC_ERR_INVALID_ARG), (4, dc.DC_OK)):
        a = dc.dc_prompt_args(0, 0.125, q.data_ptr(), k.data_ptr(), v.data_ptr(), 256, 64, 128, 64, 128, 64, out.data_ptr(),
                              lse.data_ptr() + at, None, 0)
        assert dc.lib().dc_prompt_attend(plan._p, C.byref(a), None) == status
    plan.check()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("step", [5.0, 9.0, 14.0, 14.9, 15.5, 23.5, 25.0, 70.0])
def test_maxima_that_rise_by_powers_of_two(step, dtype):
    """Every 128 keys the scores rise by a factor of 2^step in weight: references that stay, and ones that move."""
    for sign in (1, -1):
        q, k, v = inputs([900], [900], 1, 4, 64, dtype)
        q[..., 0] = 8.0
        k[:, 0, 0] = (sign * step * math.log(2) * (torch.arange(900, device="cuda") // 128)).to(dtype)
        out, lse = dc.PromptPlan([900], 1, 64, q_heads=4).attend(q, k, v, with_lse=True)
        compare(out, lse, q, k, v, [900], [900])


def test_a_fresh_plan_on_another_stream():
    """Plans made and used at once on a stream that does not wait for the default one, which is busy all the while: the
    plan has arrived when the call returns, and its making does not wait for that work."""
    import random
    r, side, plans = random.Random(3), torch.cuda.Stream(), []
    cases = [[r.randint(1, 200) for _ in range(r.choice([1, 5, 40, 300]))] for _ in range(24)]
    k_lens = [[n + r.choice([0, 300, 3000 // len(ls)]) for n in ls] for ls in cases]
    data = [inputs(a, b, 2, 2, 64, BF, seed=i) for i, (a, b) in enumerate(zip(cases, k_lens))]
    plans.append(dc.PromptPlan([1], 2, 64, q_heads=4).attend(*inputs([1], [1], 2, 2, 64, BF)))  # (what a first call sets up)
    torch.cuda.synchronize()
    outs, busy = [], torch.cuda.Event()
    torch.cuda._sleep(1 << 30)  # half a second or more
    busy.record()
    for i, (a, b) in enumerate(zip(cases, k_lens)):
        plans.append(dc.PromptPlan(a, 2, 64, q_heads=4, k_lens=b))
        if i % 2:
            with torch.cuda.stream(side):
                outs.append(plans[-1].attend(*data[i], with_lse=True))
        else:
            outs.append(plans[-1].attend(*data[i], with_lse=True, stream=side))
    side.synchronize()
    assert not busy.query(), "the default stream's work was waited for"
    torch.cuda.synchronize()
    for i, (out, lse) in enumerate(outs):
        compare(out, lse, *data[i], cases[i], k_lens[i])


def test_plans_come_and_go_during_a_capture():
    """A plan dropped while a stream captures (by the garbage collector, say), and one made and used there."""
    lens = [70, 130]
    q, k, v = inputs(lens, lens, 2, 4, 64, BF)
    old = [dc.PromptPlan([n], 2, 64, q_heads=8) for n in (5, 300)]
    want = dc.PromptPlan(lens, 2, 64, q_heads=8).attend(q, k, v)
    out, graph = torch.zeros_like(want), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        old.pop()
        plan = dc.PromptPlan(lens, 2, 64, q_heads=8)
        plan.attend(q, k, v, out=out)
        old[0].close()
    for _ in range(2):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    plan.check()


def test_rows_computed_anew_over_many_keys():
    """A NaN among the last values: all rows of the items that must not see it are computed anew, which takes over a second
    (the waits of a debug build would give up after half of one if they did not count the keys). Keys and values of the
    heads overlap in memory."""
    n, d, group, ql = 60000, 64, 4, 64
    heads = torch.cuda.get_device_properties(0).multi_processor_count  # (an item each, none in parts)
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn((ql, heads * group, d), device="cuda", generator=g).to(BF)
    kb, vb = (torch.randn(8 * (n + heads) + d, device="cuda", generator=g).to(BF) for _ in range(2))
    vb[8 * (n - 1):] = math.nan  # (of the first head's values, dims of the last eight)
    k, v = (x.as_strided((n, heads, d), (8, 8, 1)) for x in (kb, vb))
    plan = dc.PromptPlan([ql], heads, d, q_heads=heads * group, k_lens=[n])
    assert plan.workspace_bytes == 0
    out, lse = plan.attend(q, k, v, with_lse=True)
    plan.check()
    some = slice(0, 2 * group)
    compare(out[:, some], lse[:, some], q[:, some], k[:, :2], v[:, :2], [ql], [n])


@pytest.mark.parametrize("dtype", [HF, BF])
@pytest.mark.parametrize("n,bits", [(4096, -18.0), (131072, -21.6), (131072, -24.6), (131072, -25.0), (1 << 20, -24.6), (1 << 20, -25.2)])
def test_many_small_weights_beside_a_large_one(n, bits, dtype):
    """One key of weight 1 and a value of 0, n - 1 others of 2^bits each with values of 1, in items that are not divided.
    In fp16 their weights are below the normal range: each is off by 2^-30 of the largest at most."""
    rows, d = 256 * torch.cuda.get_device_properties(0).multi_processor_count, 64
    q = torch.zeros((rows, 1, d), dtype=dtype, device="cuda")
    k, v = torch.zeros((n, 1, d), dtype=dtype, device="cuda"), torch.ones((n, 1, d), dtype=dtype, device="cuda")
    q[..., 0] = 1.0
    k[: n - 1, 0, 0] = bits * math.log(2) / 0.125
    v[n - 1] = 0.0
    plan = dc.PromptPlan([rows], 1, d, q_heads=1, k_lens=[n], causal=False)
    out = plan.attend(q, k, v)
    plan.check()
    w = (n - 1) * math.exp(0.125 * float(k[0, 0, 0]))
    want = w / (1 + w)
    u = torch.finfo(dtype).eps / 2
    tol = 1.02 * 2 * u * want + (n * 2.0 ** -30 + 2.0 ** -25 if dtype == HF else 0)
    assert float((out.double() - want).abs().max()) <= tol


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("scale", [1e-30, 1.2e-38, 1e-38, 1e-39, 1e-42])
def test_the_smallest_scales(scale, dtype):
    q, k, v = inputs([300], [300], 1, 4, 64, dtype)
    out, lse = dc.PromptPlan([300], 1, 64, q_heads=4).attend(q, k, v, with_lse=True, scale=scale)
    compare(out, lse, q, k, v, [300], [300], scale=scale)
