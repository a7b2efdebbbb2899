"""Attention whose scores are far from 0: weights depend on how far a score lies below the largest alone, whatever both are.

Scores are whole numbers here, and exact in 32 bits in any order of their sums: 2^base from the first dim, `step` times a
small whole number from the others. So the results' own roundings are all that they may be off by: each weight and the
result once, u each; exponents by 2^-23 of themselves, and those of weights that count (above 2^-40) by 2^-17; in fp16 a weight
below the normal range by 2^-25 of the largest; 2^-14 of the sums for the rest."""

import math

import numpy as np
import pytest
import torch

from attention64 import U, check
from paged_plain import make_tables, tokens_of
from paper_2608_08878_gb300 import dc

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def exact64(q, k, v, seen, scale):
    """(o, lse, tolerances) of q [..., r, d], k, v [..., n, d], seen [..., r, n] in 64 bits."""
    dtype, scale = q.dtype, float(np.float32(scale))
    z = q.double() @ k.double().transpose(-1, -2)
    z = torch.where(seen, z, -math.inf)
    m = z.amax(-1, keepdim=True)
    none = m == -math.inf
    p = torch.where(seen, torch.exp((z - torch.where(none, 0.0, m)) * scale), 0.0)
    l = p.sum(-1, keepdim=True)
    w = p / torch.where(none, 1.0, l)
    o, size = w @ v.double(), w @ v.double().abs()
    lse = torch.where(none, -math.inf, m * scale + torch.log(l)).squeeze(-1)
    tol = 1.02 * U[dtype] * (size + o.abs()) + 2.0 ** -14 * size + 1e-30
    if dtype == HF:
        tol = tol + 2.0 ** -25 * (1 + k.shape[-2] * v.double().abs().amax(-2, keepdim=True))
    finite = torch.where(torch.isfinite(lse), lse, 0.0)
    return o, lse, tol, 2.0 ** -22 * finite.abs() + 2.0 ** -20


def parts(base, step):
    """2^base and step as products of two numbers that both types have."""
    a = base // 2
    s = int(math.log2(step)) // 2
    return 2.0 ** a, 2.0 ** (base - a), 2.0 ** s, step / 2.0 ** s


def tokens(shape, g, first, rest):
    x = torch.randint(-1, 2, shape, device="cuda", generator=g).float() * rest
    x[..., 0] = first
    return x


KINDS = [(20, 1, 0.5), (20, 1, 8.0), (20, 1, 4096.0), (20, 1, 1e9), (20, 1, 1e30), (22, 2, 0.125), (0, 1, 1e7), (-20, 1, 1.0),
         (29, 1024, 0.088388)]


def filled(lens, page, kvh, group, d, dtype, base, step, common=()):
    """A cache with such keys, queries with such scores; where base is below 0 so are the scores, around -2^-base."""
    sign = 1.0 if base >= 0 else -1.0
    a, b, s, t = parts(abs(base), step)
    if base == 0:
        a = b = 0.0
    tables, pool = make_tables(lens, page, common=common)
    cache = dc.PagedCache(1, pool, kvh, d, page_size=page, q_heads=kvh * group, dtype=dtype)
    g = torch.Generator(device="cuda").manual_seed(7)
    cache.k[0].copy_(tokens(cache.k[0].shape, g, b, t))
    cache.v[0].copy_(torch.randn(cache.v[0].shape, device="cuda", generator=g))
    q = tokens((len(lens), kvh * group, d), g, sign * a, s).to(dtype)
    return cache, tables, torch.tensor(lens, dtype=torch.int32, device="cuda"), q


def compare(out, lse, q, cache, tables, lens, scale, pick=None):
    for s, n in enumerate(lens):
        x = q[s].view(cache.kv_heads, -1, cache.head_dim)
        k, v = tokens_of(cache.k[0], tables, s, n), tokens_of(cache.v[0], tables, s, n)
        seen = torch.ones((cache.kv_heads, 1, n), dtype=torch.bool, device="cuda")
        if pick is not None:
            on = torch.zeros_like(seen)
            for h in range(cache.kv_heads):
                for j in pick[s, h].tolist():
                    if j >= 0:
                        on[h, 0, j * cache.page_size: (j + 1) * cache.page_size] = True
            seen = on
        o, z, tol, tolz = exact64(x, k, v, seen.expand(-1, x.shape[1], -1), scale)
        check(out[s].view_as(o), o, tol, f"sequence {s}")
        check(lse[s].view_as(z), z, tolz, f"sequence {s}: lse")


@pytest.mark.parametrize("base,step,scale", KINDS)
@pytest.mark.parametrize("dtype", [BF, HF])
def test_paged(base, step, scale, dtype):
    lens = [5, 700, 2100, 9000]
    cache, tables, n, q = filled(lens, 64, 2, 4, 128, dtype, base, step)
    out, lse = cache.attend(q, tables, n, scale=scale, with_lse=True)
    cache.check()
    compare(out, lse, q, cache, tables, lens, scale)
    pick = cache.select(q, tables, n, 20)
    out, lse = cache.attend(q, tables, n, scale=scale, selected=pick, with_lse=True)
    cache.check()
    compare(out, lse, q, cache, tables, lens, scale, pick)


@pytest.mark.parametrize("group,d", [(9, 64), (17, 128), (33, 64), (4, 64)])
@pytest.mark.parametrize("scale", [0.5, 1e9])
def test_paged_groups_and_whole_units(group, d, scale):
    lens = [600 - 13 * i for i in range(38)]  # (on 152 SMs these are not cut)
    cache, tables, n, q = filled(lens, 32, 4, group, d, BF, 20, 1)
    out, lse = cache.attend(q, tables, n, scale=scale, with_lse=True)
    cache.check()
    compare(out, lse, q, cache, tables, lens, scale)


@pytest.mark.parametrize("base,step,scale", KINDS)
@pytest.mark.parametrize("dtype,d", [(BF, 128), (HF, 64), (HF, 128)])
def test_paged_shared(base, step, scale, dtype, d):
    common = [(0, 3, 2048), (3, 40, 160)]
    lens = [2048 + x for x in (0, 7, 300)] + [160 + (i * 37) % 200 for i in range(40)] + [333]
    cache, tables, n, q = filled(lens, 32, 2, 4, d, dtype, base, step, common)
    out, lse = cache.attend(q, tables, n, scale=scale, shared=cache.share([3, 40], [2048, 160]), with_lse=True)
    cache.check()
    compare(out, lse, q, cache, tables, lens, scale)


@pytest.mark.parametrize("base,step,scale", KINDS)
@pytest.mark.parametrize("dtype,d", [(BF, 128), (HF, 64), (HF, 128), (BF, 64)])
def test_prompts(base, step, scale, dtype, d):
    q_lens, k_lens, kvh, group = [1, 300, 40], [5000, 300, 170], 2, 4
    sign = 1.0 if base >= 0 else -1.0
    a, b, s, t = parts(abs(base), step)
    if base == 0:
        a = b = 0.0
    g = torch.Generator(device="cuda").manual_seed(8)
    q = tokens((sum(q_lens), kvh * group, d), g, sign * a, s).to(dtype)
    k = tokens((sum(k_lens), kvh, d), g, b, t).to(dtype)
    v = torch.randn(k.shape, device="cuda", generator=g).to(dtype)
    if base == 0:  # a value that is not finite, where rows must not see it
        v[-1, 1, 3] = math.nan
    plan = dc.PromptPlan(q_lens, kvh, d, q_heads=kvh * group, k_lens=k_lens)
    out, lse = plan.attend(q, k, v, scale=scale, with_lse=True)
    plan.check()
    q0 = k0 = 0
    for ql, kl in zip(q_lens, k_lens):
        x = q[q0: q0 + ql].view(ql, kvh, group, d).permute(1, 2, 0, 3)
        kk, vv = (y[k0: k0 + kl].transpose(0, 1)[:, None] for y in (k, v))
        seen = torch.arange(kl, device="cuda") <= torch.arange(ql, device="cuda")[:, None] + kl - ql
        last = torch.isnan(vv.float()).any()
        o, z, tol, tolz = exact64(x, kk, torch.nan_to_num(vv), seen.expand(kvh, group, ql, kl), scale)
        got = out[q0: q0 + ql].view(ql, kvh, group, d).permute(1, 2, 0, 3)
        zz = lse[q0: q0 + ql].view(ql, kvh, group).permute(1, 2, 0)
        if last:  # (only the last row sees that value)
            assert bool(torch.isfinite(got[:, :, :-1]).all())
            o, tol, got = o[:, :, :-1], tol[:, :, :-1], got[:, :, :-1]
        check(got, o, tol)
        check(zz, z, tolz, "lse")
        q0, k0 = q0 + ql, k0 + kl


@pytest.mark.parametrize("dtype,d", [(BF, 128), (HF, 64)])
@pytest.mark.parametrize("scale", [1e38, 3e38])
def test_prompts_at_the_largest_scales(scale, dtype, d):
    """scale times log2(e) is past what 32 bits hold: the keys of the largest score share the weight."""
    g = torch.Generator(device="cuda").manual_seed(10)
    n, kvh, group = 300, 2, 4
    q = torch.randint(-1, 2, (n, kvh * group, d), device="cuda", generator=g).to(dtype)
    k = torch.randint(-1, 2, (n, kvh, d), device="cuda", generator=g).to(dtype)
    v = torch.randn((n, kvh, d), device="cuda", generator=g).to(dtype)
    plan = dc.PromptPlan([n], kvh, d, q_heads=kvh * group)
    out = plan.attend(q, k, v, scale=scale)
    plan.check()
    x = q.view(n, kvh, group, d).permute(1, 2, 0, 3)
    seen = torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
    o, _, tol, _ = exact64(x, k.transpose(0, 1)[:, None], v.transpose(0, 1)[:, None], seen.expand(kvh, group, n, n), scale)
    check(out.view(n, kvh, group, d).permute(1, 2, 0, 3), o, tol)


@pytest.mark.parametrize("base,step", [(20, 1), (29, 2 ** 10), (39, 2 ** 19), (39, 2 ** 20)])
@pytest.mark.parametrize("n", [130, 3000])
def test_trees(base, step, n):
    kvh, group, d, T = 2, 4, 128, 12
    cache = dc.DistillCache(1, kvh, d, n + 40, n, batch=2, q_heads=kvh * group)
    a, b, s, t = parts(base, step)
    g = torch.Generator(device="cuda").manual_seed(9)
    k = tokens((1, 2, kvh, n, d), g, b, t).to(BF)
    v = torch.randn(k.shape, device="cuda", generator=g).to(BF)
    cache.append(k, v)
    q = tokens((1, 2, T, kvh * group, d), g, a, s).to(BF)
    kd = tokens((1, 2, kvh, T, d), g, b, t).to(BF)
    vd = torch.randn(kd.shape, device="cuda", generator=g).to(BF)
    parents = (torch.arange(T, dtype=torch.int32, device="cuda") - 1).expand(2, T).contiguous()
    out = cache.tree_attend(q, kd, vd, parents)
    cache.sync()
    seen = torch.cat([torch.ones((T, n), dtype=torch.bool, device="cuda"), torch.ones((T, T), dtype=torch.bool, device="cuda").tril()], 1)
    x = q[0].view(2, T, kvh, group, d).permute(0, 2, 3, 1, 4)
    kk, vv = torch.cat([k[0], kd[0]], 2)[:, :, None], torch.cat([v[0], vd[0]], 2)[:, :, None]
    o, _, tol, _ = exact64(x, kk, vv, seen.expand(2, kvh, group, T, n + T), d ** -0.5)
    check(out[0].view(2, T, kvh, group, d).permute(0, 2, 3, 1, 4), o, tol)
