"""Drafted trees over rows of very different lengths (per-row budgets): short rows among long ones in every order, several
pairs of query tiles, rows in parts, and what lies past a short row's end."""

import math
import random

import pytest
import torch

from paper_2608_08878_gb300 import dc
from test_gpu_tree import BF, compare, make, rand, tree

pytestmark = pytest.mark.gpu


def budgets_of(kind, rows, n, seed=0):
    r = random.Random(seed)
    if kind == "apart":      # a long row in five
        return [n if i % 5 == 0 else max(1, n // 16) for i in range(rows)]
    if kind == "adjacent":   # the long ones together
        return [n if i < (rows + 4) // 5 else max(1, n // 16) for i in range(rows)]
    if kind == "ones":       # one long row, the others of one token
        return [n if i == rows // 2 else 1 for i in range(rows)]
    if kind == "last":
        return [n if i == rows - 1 else 1 + i % 130 for i in range(rows)]
    return [max(1, min(n, int(2 ** r.uniform(0, math.log2(n + 1))))) for _ in range(rows)]


def uneven(layers, batch, kvh, group, d, n, T, kind, bad=None, tree_kind="random", seed=0):
    """A cache whose rows keep those budgets; `bad`: the slots past their ends hold values of that kind."""
    rows = layers * batch * kvh
    budgets = budgets_of(kind, rows, n, seed)
    cache, draft = make(layers, batch, kvh, group, d, n, T, kind=tree_kind, seed=seed, **(dict(scorer=2, n_sinks=n) if bad else {}))
    one = lambda s: (rand(layers, batch, kvh * group, d, seed=s), rand(layers, batch, kvh, d, seed=s + 1),  # noqa: E731
                     rand(layers, batch, kvh, d, seed=s + 2))
    cache.set_row_budgets(budgets)
    cache.decode_step(*one(seed + 30))
    cache.evict()
    if bad:  # (the sinks stay, what comes later goes)
        k, v = (torch.full((layers, batch, kvh, 30, d), bad, dtype=BF, device="cuda") for _ in range(2))
        cache.append(k, v)
        cache.decode_step(*one(seed + 40))
        cache.evict()
    assert list(cache.row_lengths()) == [min(b, n + 1) for b in budgets]
    return cache, draft


SHAPES = [(2, 1, 4, 8, 128, 3000, 100), (4, 4, 8, 4, 64, 700, 16), (5, 4, 8, 8, 128, 900, 128), (5, 8, 8, 4, 128, 410, 8),
          (1, 1, 8, 4, 128, 20000, 3), (19, 2, 4, 2, 64, 2100, 70), (1, 1, 3, 8, 64, 5000, 1)]


@pytest.mark.parametrize("kind", ["apart", "adjacent", "ones", "last", "random"])
@pytest.mark.parametrize("shape", SHAPES)
def test_rows_of_different_lengths(shape, kind):
    cache, draft = uneven(*shape, kind)
    out = cache.tree_attend(*draft)
    cache.sync()
    compare(cache, draft, out)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("shape", [(2, 1, 4, 8, 128, 3000, 100), (5, 8, 4, 4, 64, 410, 8), (1, 1, 8, 4, 128, 5000, 3)])
def test_slots_past_a_short_rows_end_hold_anything(shape, bad):
    for kind in ("apart", "last", "random"):
        cache, draft = uneven(*shape, kind, bad)
        out = cache.tree_attend(*draft)
        cache.sync()
        assert bool(torch.isfinite(out.float()).all())
        compare(cache, draft, out)


def test_rows_of_no_token():
    """Per-row budgets on a cache that holds nothing yet: the drafts alone."""
    cache = dc.DistillCache(2, 2, 64, 300, 100, batch=2, q_heads=8)
    cache.set_row_budgets([100, 3, 7, 50, 1, 1, 100, 9])
    draft = (rand(2, 2, 6, 8, 64), rand(2, 2, 2, 6, 64, seed=1), rand(2, 2, 2, 6, 64, seed=2), tree(2, 6, "random"))
    compare(cache, draft, cache.tree_attend(*draft))
    cache.sync()


def test_random_rows():
    r = random.Random(9)
    for i in range(24):
        uneven_shape = (r.choice([1, 2, 5, 12]), r.choice([1, 3, 8]), r.choice([1, 2, 8]), r.choice([1, 2, 4, 8]), r.choice([64, 128]),
                        int(2 ** r.uniform(0, 12)) + 1, min(128, int(2 ** r.uniform(0, 7.2))))
        cache, draft = uneven(*uneven_shape, r.choice(["apart", "adjacent", "ones", "last", "random"]),
                              tree_kind=r.choice(["random", "chain", "flat", "holes"]), seed=i)
        out = cache.tree_attend(*draft)
        cache.sync()
        compare(cache, draft, out)


@pytest.mark.parametrize("kw", [dict(global_tokens=True), dict(scorer=1), dict(scorer=2), dict(alpha_mode=1), dict(engine=1),
                                dict(budget_ratio=0.3)])
def test_caches_of_every_kind(kw):
    cache, draft = make(2, 2, 2, 4, 128, 700, 20, **kw)
    for i in range(3):
        cache.step(rand(2, 2, 8, 128, seed=8 + i), rand(2, 2, 2, 128, seed=19 + i), rand(2, 2, 2, 128, seed=30 + i), budget=300 - 50 * i)
        compare(cache, draft, cache.tree_attend(*draft))
    cache.sync()


@pytest.mark.parametrize("kw", [dict(), dict(engine=1), dict(global_tokens=True), dict(scorer=1)])
def test_steps_are_the_same_with_trees_between(kw):
    """Before a step and between a step's scores and its eviction, with rows in parts: all results and the cache bit for bit."""
    runs = []
    for between in (False, True):
        cache, draft = make(2, 2, 4, 4, 128, 3000, 12, **kw)
        got = []
        for i in range(6):
            x = (rand(2, 2, 16, 128, seed=8 + i), rand(2, 2, 4, 128, seed=90 + i), rand(2, 2, 4, 128, seed=50 + i))
            if between:
                cache.tree_attend(*draft)
            if i % 2:
                got.append(cache.step(*x, budget=2000 - i))
                continue
            got.append(cache.decode_step(*x))
            if between:
                cache.tree_attend(*draft)
            cache.evict(2000 - i)
        cache.sync()
        runs.append(got + [cache.buffer(b)[:, :1995] for b in (dc.BUF_K, dc.BUF_V, dc.BUF_POS)])
    assert all(torch.equal(a, b) for a, b in zip(*runs))
