"""Long rows of prompt and tree attention with values that mark their key tiles: work that is lost or done twice
between the parts of a row shows, where the mean of many random values would hide it."""

import pytest
import torch

import test_gpu_prompt as prompts
import test_gpu_tree as trees
from attention64 import attention64, check
from marks import marked
from paper_2608_08878_gb300 import dc

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


@pytest.mark.parametrize("q_lens,k_lens,kvh,group,d,dtype", [
    ([1] * 6, [20000, 1, 127, 128, 129, 4097], 8, 4, 128, BF), ([1], [50001], 1, 8, 64, BF), ([2, 1], [33333, 3], 1, 1, 128, HF),
    ([1] * 3, [70001, 30000, 9], 2, 4, 64, HF), ([300, 77], [9000, 40001], 2, 4, 128, BF), ([8192], [8192], 2, 4, 128, BF),
    ([4099, 4097], [4099, 4097], 1, 8, 64, HF), ([512] * 20, [512 + 300 * i for i in range(20)], 4, 8, 128, BF)])
@pytest.mark.parametrize("causal", [True, False])
def test_every_key_tile_of_a_prompt(q_lens, k_lens, kvh, group, d, dtype, causal):
    q, k, v = prompts.inputs(q_lens, k_lens, kvh, group, d, dtype)
    at = 0
    for s, n in enumerate(k_lens):
        for h in range(kvh):
            v[at: at + n, h] = marked(n, d, dtype, "cuda", 17 * (s * kvh + h))
        at += n
    plan = dc.PromptPlan(q_lens, kvh, d, q_heads=kvh * group, k_lens=k_lens, causal=causal)
    out, lse = plan.attend(q, k, v, with_lse=True)
    plan.check()
    prompts.compare(out, lse, q, k, v, q_lens, k_lens, causal, rows=256)


def tree_of_marks(layers, batch, kvh, group, d, n, T, part=0, parts=1):
    cache = dc.DistillCache(layers, kvh, d, n + 8, max(1, n - 1), batch=batch, q_heads=kvh * group, window=1)
    shape = (layers, batch, kvh, n, d)
    k = torch.empty(shape, dtype=BF, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    v = torch.empty(shape, dtype=BF, device="cuda")
    kd, vd = trees.rand(layers, batch, kvh, T, d, seed=2), torch.zeros((layers, batch, kvh, T, d), dtype=BF, device="cuda")
    for r in range(layers * batch * kvh):
        v.view(-1, n, d)[r] = marked(n, d, BF, "cuda", 17 * r, part, parts)
        vd.view(-1, T, d)[r, :, (29 * r + 5) % d] = 4096.0 / T
    cache.append(k, v)
    return cache, (trees.rand(layers, batch, T, kvh * group, d, seed=3), kd, vd, trees.tree(batch, T, "random", 4))


@pytest.mark.parametrize("shape", [
    (1, 1, 2, 4, 128, 30000, 9), (1, 1, 1, 1, 64, 70001, 1), (1, 2, 4, 8, 128, 20000, 64), (1, 1, 3, 4, 64, 40000, 100),
    (2, 19, 4, 4, 128, 4097, 16), (1, 151, 1, 4, 64, 2048, 8), (1, 7, 1, 8, 128, 9999, 40), (3, 51, 1, 2, 128, 1500, 3)])
def test_every_key_tile_of_a_row(shape):
    cache, draft = tree_of_marks(*shape)
    out = cache.tree_attend(*draft)
    cache.sync()
    trees.compare(cache, draft, out)


@pytest.mark.parametrize("part", range(8))
def test_every_key_tile_past_32_bits(part):
    """The last row's keys lie past 2^32 bytes into the cache's, 17969 tiles a row, an eighth of them marked at a time; and
    what the comparison would not let by."""
    n, d, T = 2_300_000, 128, 3
    cache, (q, kd, vd, parents) = tree_of_marks(1, 1, 8, 1, d, n, T, part, 8)
    out = cache.tree_attend(q, kd, vd, parents)
    cache.sync()
    K, V, anc = cache.buffer(dc.BUF_K), cache.buffer(dc.BUF_V), trees.masks(parents)
    for r in (0, 3, 7):
        seen = torch.cat([torch.ones((T, n), dtype=torch.bool, device="cuda"), anc[0]], 1)
        kk, vv = torch.cat([K[r, :n], kd[0, 0, r]]), torch.cat([V[r, :n], vd[0, 0, r]])
        o, _, tol, _ = attention64(q[0, 0, :, r], kk, vv, seen, d ** -0.5)
        check(out[0, 0, :, r], o, tol, f"row {r}")
        if r == 7:
            for lost in ((part * d), (part * d + 8 * d * 8 + 77), (part * d + 8 * d * 16 + 100)):  # (a whole tile)
                seen[:, lost * 128: lost * 128 + 128] = False
                less = attention64(q[0, 0, :, r], kk, vv, seen, d ** -0.5)[0]
                with pytest.raises(AssertionError):
                    check(less, o, tol)
                seen[:, lost * 128: lost * 128 + 128] = True
