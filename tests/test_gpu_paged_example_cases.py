"""examples/paged_samples.py at its smallest and largest numbers of pages, with prompts that end with a page and with short ones,
and its selected attention against the plain one."""

import pytest
import torch

from attention64 import check
from paged_plain import attend64, plain_select
from test_gpu_paged_example import example

pytestmark = pytest.mark.gpu


def same_as_in_one_pass(m, out, prompt, logits, model):
    for i in range(len(out)):
        text = torch.cat([prompt, out[i, :-1]])
        n = len(text)
        pages = -(-n // 32)
        cache = m.dc.PagedCache(len(model.layers), pages, model.kvh, model.d, page_size=32, q_heads=model.hq)
        tables = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1)
        keys = torch.empty((n, model.kvh, model.d), dtype=torch.bfloat16, device="cuda")
        plan = m.dc.PromptPlan([n], model.kvh, model.d, q_heads=model.hq)
        want = model.forward(text, cache, tables, torch.zeros(1, dtype=torch.int32, device="cuda"),
                             lambda j, q, k, v: plan.attend(q, k, v), k_out=keys)[-1].float()
        # (as in test_gpu_paged_example.py: a few roundings of 2^-9 a layer)
        assert float((logits[i].float() - want).norm() / want.norm()) < 16 * 2.0 ** -9


@pytest.mark.parametrize("prompt_len", [1, 31, 32, 33, 192])
@pytest.mark.parametrize("tokens", [1, 2, 9])
@pytest.mark.parametrize("pages", [0, 20])
def test_all_pages(prompt_len, tokens, pages):
    m = example()
    out, prompt, logits, model = m.run(samples=2, tokens=tokens, pages=pages, prompt_len=prompt_len)
    assert out.shape == (2, tokens) and len(prompt) == prompt_len
    same_as_in_one_pass(m, out, prompt, logits, model)


@pytest.mark.parametrize("pages", [1, 2, 3, 5])
@pytest.mark.parametrize("prompt_len", [20, 224, 300])
def test_selected_pages(pages, prompt_len, monkeypatch):
    m = example()
    seen = []
    select, attend = m.dc.PagedCache.select, m.dc.PagedCache.attend

    def checked_select(cache, q, tables, lens, count, **kw):
        got = select(cache, q, tables, lens, count, **kw)
        if not torch.cuda.is_current_stream_capturing():
            want = plain_select(q, cache.bounds[kw["layer"]], tables, lens.tolist(), cache.page_size, count, kw["keep_first"],
                                kw["keep_last"])
            assert torch.equal(got, want)
        return got

    def checked_attend(cache, q, tables, lens, **kw):
        out = attend(cache, q, tables, lens, **kw)
        if not torch.cuda.is_current_stream_capturing():
            sel, layer = kw.get("selected"), kw["layer"]
            o, _, tol, _ = attend64(q, cache.k[layer], cache.v[layer], tables, lens.tolist(), selected=sel)
            check(out, o, tol)
            if sel is not None:
                assert lens.tolist() == [prompt_len + 1] * len(lens)  # the newest token among them
                last = (prompt_len + cache.page_size) // cache.page_size - 1
                assert bool((sel == last).any(-1).all())
                seen.append(layer)
        return out

    monkeypatch.setattr(m.dc.PagedCache, "select", checked_select)
    monkeypatch.setattr(m.dc.PagedCache, "attend", checked_attend)
    out, _, logits, model = m.run(samples=3, tokens=40, pages=pages, prompt_len=prompt_len)
    assert seen == [0, 1] and out.shape == (3, 40)
    assert 0 <= int(out.min()) and int(out.max()) < model.vocab and bool(torch.isfinite(logits.float()).all())


@pytest.mark.parametrize("kw", [dict(samples=0), dict(tokens=0), dict(pages=-1), dict(prompt_len=0)])
def test_refuses(kw):
    with pytest.raises(ValueError):
        example().run(**kw)


def test_command_line(monkeypatch, capsys):
    m = example()
    for argv, fine in ((["--pages", "1", "--tokens", "3"], True), (["--pages", "2", "--tokens", "1", "--samples", "2"], True),
                       (["--tokens", "0"], False), (["--pages", "-1"], False), (["--samples", "0"], False)):
        monkeypatch.setattr("sys.argv", ["paged_samples.py"] + argv)
        if fine:
            m.main()
            assert "sample 1:" in capsys.readouterr().out
        else:
            with pytest.raises(SystemExit):
                m.main()
