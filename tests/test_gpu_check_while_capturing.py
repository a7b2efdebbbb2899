"""`check` of a paged cache and of a prompt plan while a stream captures: the capture is kept, the check says what it should."""

import threading

import pytest
import torch

from paper_2608_08878_gb300 import dc
from test_gpu_paged import filled

pytestmark = pytest.mark.gpu


def checked():
    cache, tables, n, q = filled([300, 70], 32, 2, 4, 64)
    plan = dc.PromptPlan([70], 2, 64, q_heads=8)
    k = torch.randn((70, 2, 64), device="cuda").to(torch.bfloat16)
    plan.attend(torch.randn((70, 8, 64), device="cuda").to(torch.bfloat16), k, k)
    return cache, tables, n, q, plan


def test_by_another_thread():
    cache, tables, n, q, plan = checked()
    want = cache.attend(q, tables, n)
    torch.cuda.synchronize()
    began, done, failed = threading.Event(), threading.Event(), []

    def check():
        try:
            began.wait(20)
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(3):
                    cache.check()
                    plan.check()
        except Exception as e:
            failed.append(e)
        finally:
            done.set()

    t = threading.Thread(target=check)
    t.start()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = cache.attend(q, tables, n)
        began.set()
        assert done.wait(20)
    t.join()
    assert not failed, failed
    out.zero_()
    graph.replay()
    assert torch.equal(out, want)


def test_of_another_stream_by_the_capturing_thread():
    cache, tables, n, q, plan = checked()
    want = cache.attend(q, tables, n)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = cache.attend(q, tables, n)
        cache.check(stream=side)
        plan.check(stream=side)
    graph.replay()
    assert torch.equal(out, want)


def test_of_the_capturing_stream_is_refused():
    cache, tables, n, q, plan = checked()
    want = cache.attend(q, tables, n)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = cache.attend(q, tables, n)
        for x in (cache, plan):
            with pytest.raises(dc.DCError) as e:
                x.check()
            assert e.value.status == dc.DC_ERR_INVALID_ARG and "captur" in str(e.value)
    graph.replay()
    assert torch.equal(out, want)
    cache.check()
    plan.check()


def test_what_a_kernel_reported():
    cache, tables, n, q, plan = checked()
    tables[0, 1] = -1
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.attend(q, tables, n)
    cache.check()
    graph.replay()
    with pytest.raises(dc.DCError) as e:
        cache.check()
    assert e.value.status == dc.DC_ERR_DEVICE
