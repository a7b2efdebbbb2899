"""Norms and rotation of queries and keys against 64 bits."""

import math

import pytest
import torch

from attention64 import U
from paper_2608_08878_gb300 import dc

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def inputs(T, hq, hk, d, rot, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randn((T, hq, d), device="cuda", generator=g).to(dtype)
    k = (3 * torch.randn((T, hk, d), device="cuda", generator=g)).to(dtype)
    pos = torch.randint(0, 1 << 17, (T,), device="cuda", generator=g, dtype=torch.int32)
    f = (10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)).float()
    w = [1 + 0.2 * torch.randn(d, device="cuda", generator=g) for _ in range(2)]
    return q, k, pos, f, w


def want64(x, pos, f, w, norm, interleaved, eps=1e-6):
    """(y, tolerance): one rounding to the type, and 32-bit arithmetic before it: the norm's few roundings, and angles
    within 2^-22 (the reduced angle, its sine and cosine), of the pair's size."""
    u = U[x.dtype]
    y = x.double()
    if norm:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps)
        if w is not None:
            y = y * w.double()
    rot = 2 * f.numel()
    a = pos.double()[:, None, None] * f.double()
    c, s = a.cos(), a.sin()
    r, rest = y[..., :rot], y[..., rot:]
    p, q = (r[..., 0::2], r[..., 1::2]) if interleaved else r.chunk(2, -1)
    o = (p * c - q * s, q * c + p * s)
    size = p.abs() + q.abs()
    if interleaved:
        out, size = torch.stack(o, -1).flatten(-2), torch.stack([size, size], -1).flatten(-2)
    else:
        out, size = torch.cat(o, -1), torch.cat([size, size], -1)
    out, size = torch.cat([out, rest], -1), torch.cat([size, rest.abs()], -1)
    return out, u * out.abs() + 2.0 ** -20 * size + 2.0 ** -25


def check(got, want):
    y, tol = want
    over = (got.double() - y).abs() - tol
    assert got.shape == y.shape and float(over.max()) <= 0, float(over.max())


def run(T, hq, hk, d, rot, dtype=BF, norm=True, interleaved=False, weights=True, seed=0):
    q, k, pos, f, w = inputs(T, hq, hk, d, rot, dtype, seed)
    wq, wk = w if weights else (None, None)
    qo, ko = dc.norm_rotate(q, k, pos, f, wq, wk, norm=norm, interleaved=interleaved)
    assert qo.dtype == ko.dtype == dtype
    for x, got, ww in ((q, qo, wq), (k, ko, wk)):
        if x.numel():
            check(got, want64(x, pos, f, ww, norm, interleaved))


@pytest.mark.parametrize("T", [1, 2, 3, 7, 32, 33, 1000, 5003])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_token_counts(T, dtype):
    run(T, 32, 8, 128, 128, dtype)


@pytest.mark.parametrize("d,rot", [(16, 16), (24, 16), (64, 64), (64, 32), (72, 48), (80, 80), (96, 96), (96, 32), (128, 128),
                                   (128, 64), (128, 16), (192, 192), (192, 64), (256, 256), (256, 112)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_head_dims(d, rot, interleaved):
    run(37, 6, 2, d, rot, interleaved=interleaved)
    run(37, 6, 2, d, rot, interleaved=interleaved, norm=False, dtype=HF)


@pytest.mark.parametrize("hq,hk", [(1, 1), (1, 0), (0, 1), (0, 3), (5, 1), (7, 7), (64, 8), (3, 2)])
def test_head_counts(hq, hk):
    run(19, hq, hk, 128, 128)
    run(3000, hq, hk, 64, 64, weights=False)


def test_no_tokens():
    q, k, pos, f, w = inputs(0, 4, 2, 64, 64, BF)
    qo, ko = dc.norm_rotate(q, k, pos, f, *w)
    assert qo.shape == q.shape and ko.shape == k.shape


def test_positions_of_any_size():
    """The largest and smallest positions, negative ones, and frequencies of whole turns and more."""
    q, k, _, f, w = inputs(9, 2, 1, 64, 64, BF)
    pos = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 1 << 24, 123456789, 77, -77], dtype=torch.int32, device="cuda")
    f = f.clone()
    f[3], f[5], f[6] = 7.0, 0.0, 1e-30
    big = f.clone()
    qo, _ = dc.norm_rotate(q, k, pos, big, *w)
    y, tol = want64(q, pos, big, w[0], True, False)
    # f / 2 pi is held to 2^-50: 2^-50 * 2^31 turns at the largest position, and 64-bit angles of 1.5e10 are themselves
    # good to 2e-6
    p = (q.double().abs().amax() * 4)
    assert float(((qo.double() - y).abs() - tol - 2e-5 * p).max()) <= 0


def test_views_and_places_for_the_results():
    T, hq, hk, d = 50, 8, 2, 128
    q, k, pos, f, w = inputs(T, hq, hk, d, d, BF)
    want = dc.norm_rotate(q, k, pos, f, *w)
    fused = torch.cat([q, k, k], 1).contiguous()
    qv, kv = fused[:, :hq], fused[:, hq: hq + hk]
    got = dc.norm_rotate(qv, kv, pos, f, *w)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # keys head by head, as the cache's append takes them
    kh = torch.zeros((hk, T, d), dtype=BF, device="cuda")
    _, ko = dc.norm_rotate(qv, kv, pos, f, *w, k_out=kh.transpose(0, 1))
    assert torch.equal(kh.transpose(0, 1), want[1]) and ko.data_ptr() == kh.data_ptr()
    # in place, the rest of the projection untouched
    dc.norm_rotate(qv, kv, pos, f, *w, q_out=qv, k_out=kv)
    assert torch.equal(fused[:, :hq], want[0]) and torch.equal(fused[:, hq: hq + hk], want[1]) and torch.equal(fused[:, hq + hk:], k)


def test_zeros_and_values_that_are_not_finite():
    q, k, pos, f, w = inputs(4, 2, 1, 64, 64, BF)
    q[0] = 0
    q[1, 0, 5] = math.nan
    q[2, 1, 5] = math.inf
    qo, ko = dc.norm_rotate(q, k, pos, f, *w)
    assert bool((qo[0] == 0).all()) and bool(torch.isnan(qo[1, 0]).all()) and bool(torch.isfinite(qo[1, 1]).all())
    assert bool(torch.isnan(qo[2, 1]).any()) and bool(torch.isfinite(qo[3]).all()) and bool(torch.isfinite(ko).all())
    qo, _ = dc.norm_rotate(q, k, pos, f, norm=False)
    other = torch.ones(64, dtype=torch.bool)
    other[[5, 37]] = False
    assert bool(torch.isfinite(qo[1, 0][other]).all()) and bool(torch.isnan(qo[1, 0][~other]).all())


@pytest.mark.parametrize("interleaved", [False, True])
def test_dims_past_the_rotated_ones_keep_to_themselves(interleaved):
    q, k, pos, f, w = inputs(3, 2, 1, 96, 32, BF)
    q[0, 0, 40], q[1, 1, 95], q[2, 0, 33] = math.nan, math.inf, -math.inf
    qo, _ = dc.norm_rotate(q, k, pos, f, norm=False, interleaved=interleaved)
    assert torch.allclose(qo[..., 32:], q[..., 32:], rtol=0, atol=0, equal_nan=True)
    assert bool(torch.isfinite(qo[..., :32]).all())


def test_tiny_and_huge_heads_keep_their_norm():
    """Squares below the normal range and above 2^127 of the type's own range: bf16 heads of 1e-18 and 1e17."""
    q, k, pos, f, w = inputs(8, 2, 1, 128, 128, BF)
    for scale, eps in ((1e-15, 1e-38), (1e17, 1e-6)):
        x = (q.float() * scale).to(BF)
        qo, _ = dc.norm_rotate(x, k, pos, f, *w, eps=eps)
        check(qo, want64(x, pos, f, w[0], True, False, eps))


def test_offsets_past_32_bits():
    T, step = 70, 1 << 26
    q, k, pos, f, w = inputs(T, 1, 1, 64, 64, BF)
    buf = torch.empty(step * (T - 1) + 128, dtype=BF, device="cuda")
    qb, kb = buf.as_strided((T, 1, 64), (step, 64, 1)), buf.as_strided((T, 1, 64), (step, 64, 1), 64)
    qb.copy_(q)
    kb.copy_(k)
    want = dc.norm_rotate(q, k, pos, f, *w)
    dc.norm_rotate(qb, kb, pos, f, *w, q_out=qb, k_out=kb)
    assert torch.equal(qb, want[0]) and torch.equal(kb, want[1])


def test_other_streams_and_graphs():
    q, k, pos, f, w = inputs(100, 8, 2, 128, 128, BF)
    want = dc.norm_rotate(q, k, pos, f, *w)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = dc.norm_rotate(q, k, pos, f, *w, stream=s)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    qo, ko = torch.zeros_like(q), torch.zeros_like(k)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dc.norm_rotate(q, k, pos, f, *w, q_out=qo, k_out=ko)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])


def test_refusals():
    q, k, pos, f, w = inputs(6, 4, 2, 64, 64, BF)
    odd = torch.zeros(6 * 4 * 64 + 1, dtype=BF, device="cuda")[1:].view(6, 4, 64)
    bad = {
        "k of another type": lambda: dc.norm_rotate(q, k.half(), pos, f),
        "q in 32 bits": lambda: dc.norm_rotate(q.float(), k.float(), pos, f),
        "k one token short": lambda: dc.norm_rotate(q, k[:5], pos, f),
        "positions of another type": lambda: dc.norm_rotate(q, k, pos.long(), f),
        "positions one short": lambda: dc.norm_rotate(q, k, pos[:5], f),
        "more frequencies than pairs": lambda: dc.norm_rotate(q, k, pos, torch.cat([f, f])),
        "an odd number of pairs": lambda: dc.norm_rotate(q, k, pos, f[:7]),
        "no frequency": lambda: dc.norm_rotate(q, k, pos, f[:0]),
        "weights of another size": lambda: dc.norm_rotate(q, k, pos, f, w[0][:32].contiguous()),
        "heads off 16 bytes": lambda: dc.norm_rotate(odd, k, pos, f),
        "dims not dense": lambda: dc.norm_rotate(q.transpose(1, 2), k.transpose(1, 2), pos, f),
        "an output of another shape": lambda: dc.norm_rotate(q, k, pos, f, q_out=k),
        "an output whose elements overlap": lambda: dc.norm_rotate(q, k, pos, f, q_out=q[:1].expand(6, 4, 64)),
        "a negative eps": lambda: dc.norm_rotate(q, k, pos, f, eps=-1.0),
    }
    for what, call in bad.items():
        with pytest.raises(dc.DCError) as e:
            call()
        assert e.value.status == dc.DC_ERR_INVALID_ARG, what


@pytest.mark.parametrize("interleaved", [False, True])
def test_frequencies_of_either_sign(interleaved):
    """Negative frequencies turn the other way, as exactly: against 64 bits, as negative positions do, and back again."""
    q, k, pos, f, _ = inputs(600, 4, 2, 128, 128, HF)
    pos = pos * 16  # to 2^21
    f = f * torch.where(torch.arange(64, device="cuda") % 3 == 0, -1.0, 1.0)
    f[1], f[2], f[4] = -7.5, -1e-8, -1.0
    for x in (f, -f, -f.abs()):
        qo, ko = dc.norm_rotate(q, k, pos, x, norm=False, interleaved=interleaved)
        check(qo, want64(q, pos, x, None, False, interleaved))
        check(ko, want64(k, pos, x, None, False, interleaved))
        assert torch.equal(dc.norm_rotate(q, k, -pos, -x, norm=False, interleaved=interleaved)[0], qo)
        back = dc.norm_rotate(qo, ko, pos, -x, norm=False, interleaved=interleaved)[0]
        assert float((back.float() - q.float()).abs().max()) <= 4 * U[HF] * float(q.abs().max())
