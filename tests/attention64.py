"""Softmax attention in 64 bits with the tolerances of a kernel that holds sums and statistics in 32
bits and rounds the weights and the output to the tensors' type: what the tests of prompt and tree
attention compare with."""

import math

import torch

# Half a unit in the last place of 1: what one rounding may change a value by, relative to it.
U = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float16)}


def attention64(q, k, v, seen, scale):
    """q [..., r, d], k, v [..., n, d] (any type), seen [..., r, n] -> (o, lse, tol_o, tol_lse) in 64 bits.

    A row that sees nothing has o = 0, lse = -infinity. Values that a row does not see have no part,
    whatever they hold.

    A score is off by at most d roundings of 2^-24 of its products' absolute sum: `ds`, from the row's largest sum.
    tol_o: every weight and the result rounded once (u each): u (sum p |v| / l + |o|), 2% more for the 32-bit
    sums; the scores' error in numerator and denominator: 2 ds sum p |v| / l; in fp16 a weight below the
    normal range is off by 2^-25 where the largest is at least 1, as is a result below it.
    tol_lse: ds, and 2^-20 of the result for the sum's and the logarithm's own."""
    u = U[q.dtype]
    fp16 = q.dtype == torch.float16
    q, k, v = q.double(), k.double(), v.double()
    z = torch.where(seen, q @ k.transpose(-1, -2) * scale, -math.inf)
    m = z.amax(-1, keepdim=True) if z.shape[-1] else z.new_full(z.shape[:-1] + (1,), -math.inf)
    p = torch.where(seen, torch.exp(z - torch.where(m == -math.inf, 0.0, m)), 0.0)
    l = p.sum(-1, keepdim=True)
    empty = ~seen.any(-1, keepdim=True)
    w = p / torch.where(empty, 1.0, l)
    # (an unseen value takes no part: 0 * infinity must not either)
    bad = ~torch.isfinite(v)
    vz = torch.where(bad, 0.0, v)
    o = w @ vz
    for kind in (math.inf, -math.inf):
        o = o + torch.where((w > 0).double() @ (v == kind).double() > 0, kind, 0.0)
    o = torch.where((w > 0).double() @ torch.isnan(v).double() > 0, math.nan, o)
    lse = (torch.where(m == -math.inf, 0.0, m) + torch.log(l)).squeeze(-1)
    d = q.shape[-1]
    finite = lambda t: torch.where(torch.isfinite(t), t, 0.0)  # noqa: E731
    ds = torch.zeros_like(lse)
    if k.shape[-2]:
        ds = torch.where(seen, finite(q).abs() @ finite(k).abs().transpose(-1, -2) * scale, 0.0).amax(-1) * (d * 2.0 ** -24)
    size = w @ vz.abs()
    tol = 1.02 * u * (size + o.abs()) + 2 * ds[..., None] * size + 1e-30
    if fp16 and k.shape[-2]:
        tol = tol + 2.0 ** -25 * (1 + k.shape[-2] * vz.abs().amax(dim=-2, keepdim=True))
    tol_lse = ds + 2.0 ** -20 * (1 + finite(lse).abs())
    return o, lse, tol, tol_lse


def check(got, want, tol, what=""):
    """Every finite value within its tolerance; the others equal."""
    got = got.double()
    assert got.shape == want.shape, what
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN where the result has none, or the reverse"
    same = (got == want) | torch.isnan(want)
    assert bool(same[~fine].all()), f"{what}: infinities differ"
    over = ((got - want).abs() - tol.expand_as(want))[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, (
        f"{what}: off by up to {float((got - want).abs()[fine].max()):.3g}, {int((over > 0).sum())} values over their tolerance")
