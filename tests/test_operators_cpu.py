"""Host-side checks of the operators around the cache: argument checks that come before the device is touched."""

import ctypes as C

import numpy as np
import pytest
import torch

from paper_2608_08878_gb300 import dc


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2608_08878_gb300 import build
    build.build()


def _rotate(**kw):
    a = dc.dc_rotate_args(tokens=4, q_heads=2, kv_heads=1, head_dim=64, rotary_dim=64, norm=1, eps=1e-6, positions=64,
                          inv_freq=64, q=64, k=64, q_out=64, k_out=64, q_token_stride=128, q_head_stride=64,
                          k_token_stride=64, k_head_stride=64, q_out_token_stride=128, q_out_head_stride=64,
                          k_out_token_stride=64, k_out_head_stride=64)
    for f, v in kw.items():
        setattr(a, f, v)
    return dc.lib().dc_norm_rotate(C.byref(a), None)


@pytest.mark.parametrize("field,value", [
    ("tokens", -1), ("tokens", 1 << 40), ("q_heads", -1), ("kv_heads", 70000), ("head_dim", 60), ("head_dim", 264),
    ("head_dim", 8), ("rotary_dim", 0), ("rotary_dim", 24), ("rotary_dim", 80), ("dtype", 2), ("eps", -1.0),
    ("eps", float("nan")), ("positions", None), ("inv_freq", None), ("q", None), ("k_out", None), ("q", 72), ("k_out", 8),
    ("q_token_stride", 130), ("k_out_head_stride", 4), ("positions", 66), ("inv_freq", 65), ("q_weight", 2), ("k_weight", 67)])
def test_norm_rotate_refuses(field, value):
    assert _rotate(**{field: value}) == dc.DC_ERR_INVALID_ARG
    assert dc.lib().dc_rotate_last_error()


def test_norm_rotate_of_nothing():
    assert _rotate(tokens=0, q=None) == dc.DC_OK
    assert _rotate(q_heads=0, kv_heads=0) == dc.DC_OK
    assert dc.lib().dc_norm_rotate(None, None) == dc.DC_ERR_INVALID_ARG


@pytest.mark.parametrize("args", [
    ([], None, 8, 2, 64), ([4, -1], None, 8, 2, 64), ([4, 4], [4, -2], 8, 2, 64), ([4], None, 8, 2, 96), ([4], None, 8, 3, 64),
    ([4], None, 1, 2, 64), ([4], None, 8, 0, 64), ([4], None, 258, 2, 64), ([1 << 29, 1], None, 8, 2, 64),
    ([1], [(1 << 29) + 1], 8, 2, 64), ([2 ** 31 - 1, 2 ** 31 - 1], None, 8, 2, 64)])
def test_prompt_plan_refuses(args):
    q, k, hq, hk, d = args
    ql = np.asarray(q, dtype=np.int32)
    kl = None if k is None else np.asarray(k, dtype=np.int32).ctypes.data_as(C.c_void_p)
    p = C.c_void_p()
    st = dc.lib().dc_prompt_plan_create(ql.ctypes.data_as(C.c_void_p), kl, ql.size, hq, hk, d, 1, C.byref(p))
    assert st == dc.DC_ERR_INVALID_ARG and not p.value
    assert dc.lib().dc_prompt_last_error()


def test_null_arguments():
    L = dc.lib()
    p = C.c_void_p()
    assert L.dc_prompt_plan_create(None, None, 1, 8, 2, 64, 1, C.byref(p)) == dc.DC_ERR_INVALID_ARG
    ql = np.ones(1, dtype=np.int32)
    assert L.dc_prompt_plan_create(ql.ctypes.data_as(C.c_void_p), None, 1, 8, 2, 64, 1, None) == dc.DC_ERR_INVALID_ARG
    assert L.dc_prompt_plan_destroy(None) == dc.DC_OK
    assert L.dc_prompt_attend(None, C.byref(dc.dc_prompt_args()), None) == dc.DC_ERR_INVALID_ARG
    assert L.dc_tree_attend(None, None, None, None, None, 0, None) == dc.DC_ERR_INVALID_ARG


def test_binding_refuses_lists_of_different_lengths_and_host_tensors():
    q, k = torch.zeros((4, 8, 64), dtype=torch.bfloat16), torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    pos, f = torch.zeros(4, dtype=torch.int32), torch.zeros(32)
    for call in (lambda: dc.PromptPlan([4], 2, 64, k_lens=[4, 4]), lambda: dc.norm_rotate(q, k, pos, f),
                 lambda: dc.norm_rotate(q.float(), k.float(), pos, f), lambda: dc.norm_rotate(q.numpy, k, pos, f)):
        with pytest.raises(dc.DCError) as e:
            call()
        assert e.value.status == dc.DC_ERR_INVALID_ARG


def test_argument_structs_match_the_header(tmp_path):
    """The header's structs have the binding's size and field offsets."""
    import os
    import shutil
    import subprocess
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    structs = {"dc_rotate_args": dc.dc_rotate_args, "dc_prompt_args": dc.dc_prompt_args}
    lines = [f'  printf("%zu\\n", sizeof({n}));' for n in structs]
    lines += [f'  printf("%zu\\n", offsetof({n}, {f}));' for n, s in structs.items() for f, _ in s._fields_]
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include "distillcache.h"\nint main(void) {\n' + "\n".join(lines) + "\n  return 0;\n}\n")
    subprocess.run([cc, "-std=c11", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "s")],
                   check=True, capture_output=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "s")], check=True, capture_output=True, text=True).stdout.split()]
    want = [C.sizeof(s) for s in structs.values()] + [getattr(s, f).offset for s in structs.values() for f, _ in s._fields_]
    assert got == want


def test_the_plain_attention_in_64_bits():
    """The tests' own reference: weights by torch's softmax, rows that see nothing, unseen values that are not finite."""
    import os
    import sys
    sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
    from attention64 import U, attention64, check
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(s, generator=g).to(torch.bfloat16) for s in ((2, 5, 8), (2, 7, 8), (2, 7, 8)))
    seen = torch.rand((2, 5, 7), generator=g) < 0.5
    seen[0, 1] = False
    seen[:, :, 3] = False
    v[:, 3] = float("nan")
    o, lse, tol, tol_lse = attention64(q, k, v, seen, 0.3)
    z = (q.double() @ k.double().transpose(1, 2) * 0.3).masked_fill(~seen, -float("inf"))
    w = torch.nan_to_num(torch.softmax(z, -1))
    vz = torch.nan_to_num(v.double())
    assert torch.allclose(o, w @ vz, atol=1e-12) and torch.allclose(lse, torch.logsumexp(z, -1)) and bool((o[0, 1] == 0).all())
    x = torch.randn(100000, generator=g, dtype=torch.float64)
    for t, u in U.items():  # one rounding stays within u, and comes near it
        off = ((x.to(t).double() - x) / x).abs()[x.abs() > 2.0 ** -10].max()
        assert 0.99 * u < float(off) <= u
    p = w.to(torch.bfloat16).double()  # weights rounded once, then the result
    check((p @ vz).to(torch.bfloat16), o, tol)
    with pytest.raises(AssertionError):
        check((p @ vz * 1.02).to(torch.bfloat16), o, tol)
    with pytest.raises(AssertionError):
        check(torch.full_like(o, float("nan")), o, tol)


def test_the_order_of_a_tensors_dimensions():
    """Drafts [layers][batch][kv_heads][nodes][d]: that shape and views of it; nodes and heads the other way round are refused."""
    shape = (2, 3, 4, 8, 64)
    for got in (shape, (6, 4, 8, 64), (24, 8, 64), (24, 512), (2 * 3 * 4 * 8 * 64,), (2, 3, 2, 2, 8, 64), (2, 3, 4, 8, 2, 32)):
        dc._order(torch.empty(got, device="meta"), "k_draft", shape)
    for got in ((2, 3, 8, 4, 64), (6, 8, 4, 64), (2, 3, 4, 64, 8), (3, 2, 4, 8, 64), (2, 3, 8, 2, 2, 64)):
        with pytest.raises(dc.DCError) as e:
            dc._order(torch.empty(got, device="meta"), "k_draft", shape)
        assert e.value.status == dc.DC_ERR_INVALID_ARG, got
    dc._order(torch.empty((6, 5, 2, 4, 64), device="meta"), "q", (2, 3, 5, 8, 64), (6, 5, 2, 4, 64))
    dc._order(torch.empty((2, 3, 0, 8, 64), device="meta"), "q", (2, 3, 0, 8, 64))


@pytest.mark.parametrize("bad", [np.asarray([2 ** 32 + 5]), [4, 2 ** 31], [-2 ** 31 - 1], [4.7], [float("nan")], [float("inf"), 3],
                                 np.asarray([2 ** 63 + 8], dtype=np.uint64), ["4"], [None], [2 ** 70]])
def test_lengths_that_int32_does_not_hold_are_refused(bad):
    for call in (lambda: dc.PromptPlan(bad, 2, 64), lambda: dc.PromptPlan([3] * len(bad), 2, 64, k_lens=bad)):
        with pytest.raises(dc.DCError) as e:
            call()
        assert e.value.status == dc.DC_ERR_INVALID_ARG


def test_lengths_of_any_whole_type():
    for x in ([5, 0, 300], np.asarray([5, 0, 300]), (5.0, 0.0, 300.0), np.asarray([5, 0, 300], dtype=np.uint16),
              torch.tensor([5, 0, 300]), torch.tensor([5, 0, 300], dtype=torch.int32), np.asarray([[5, 0, 300]])):
        got = dc._lengths(x, "q_lens")
        assert got.dtype == np.int32 and got.flags.c_contiguous and got.tolist() == [5, 0, 300]
    assert dc._lengths([], "q_lens").size == 0


@pytest.mark.parametrize("lens,hq,hk", [([1 << 29], 65535 * 128, 65535), ([1] * 20000, 65535, 65535), ([1 << 22] * 3, 65535 * 8, 65535)])
def test_more_work_than_a_plan_counts_is_refused(lens, hq, hk):
    """Items are numbered by ints and take 64 bytes each on the host and the device: refused before any is made."""
    ql = np.asarray(lens, dtype=np.int32)
    p = C.c_void_p()
    st = dc.lib().dc_prompt_plan_create(ql.ctypes.data_as(C.c_void_p), None, ql.size, hq, hk, 64, 1, C.byref(p))
    assert st == dc.DC_ERR_INVALID_ARG and not p.value and b"items" in dc.lib().dc_prompt_last_error()


@pytest.mark.parametrize("n,d,dtype", [(20000, 128, torch.bfloat16), (30000, 128, torch.bfloat16), (50001, 64, torch.bfloat16),
                                       (70001, 64, torch.bfloat16), (33333, 128, torch.float16)])
def test_marked_values_show_a_tile_that_is_lost_or_read_twice(n, d, dtype):
    """The comparison of long rows with values of marked() does not let one whole key tile of 128 by, wherever it is."""
    import os
    import sys
    sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
    from attention64 import attention64, check
    from marks import marked
    g = torch.Generator().manual_seed(n)
    q, k = (torch.randn(s, generator=g).to(dtype) for s in ((2, d), (n, d)))
    v = marked(n, d, dtype, "cpu", 5)
    seen = torch.ones((2, n), dtype=torch.bool)
    o, _, tol, _ = attention64(q, k, v, seen, d ** -0.5)
    check(o.to(dtype), o, tol)
    tiles = n // 128
    for t in {0, 1, tiles // 2, tiles - 1} | set(torch.randint(0, tiles, (4,), generator=g).tolist()):
        at = slice(t * 128, t * 128 + 128)
        seen[:, at] = False
        less = attention64(q, k, v, seen, d ** -0.5)[0]
        seen[:, at] = True
        twice = attention64(q, torch.cat([k, k[at]]), torch.cat([v, v[at]]), torch.ones((2, n + 128), dtype=torch.bool), d ** -0.5)[0]
        for wrong in (less, twice):
            with pytest.raises(AssertionError):
                check(wrong.to(dtype), o, tol)
