"""Several samples of one prompt over a paged cache, on a toy model with random weights.

The prompt goes through the model once: its keys and values into pages (`dc.PagedCache.append`), its own attention by
`dc.PromptPlan`. Every sample's table then begins with the prompt's pages, which are stored and read once for all of
them (`share`), and goes on with pages of its own. A step appends one token to each sample and attends over all
that it has (dense), or over the few pages that can matter most to it (`select`), with the step captured
into a CUDA graph once and replayed: lengths, tables and tokens are on the device.

    python examples/paged_samples.py [--samples N] [--tokens N] [--pages N]
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_08878_gb300 import dc  # noqa: E402

BF = torch.bfloat16


class ToyModel:
    """layers of attention between an embedding and an output matrix."""

    def __init__(self, layers=2, kv_heads=2, group=4, d=64, vocab=256, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.kvh, self.hq, self.d, self.vocab, dim = kv_heads, kv_heads * group, d, vocab, kv_heads * group * d
        rand = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
        self.embed, self.head = rand(vocab, dim).to(BF), (rand(dim, vocab) / dim ** 0.5).to(BF)
        self.layers = [dict(qkv=(rand(dim, (self.hq + 2 * kv_heads) * d) / dim ** 0.5).to(BF),
                            out=(rand(dim, dim) / dim ** 0.5).to(BF), wq=1 + 0.1 * rand(d), wk=1 + 0.1 * rand(d)) for _ in range(layers)]
        self.inv_freq = (10000.0 ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)).float()

    def forward(self, tokens, cache, tables, lens, attend, starts=None, k_out=None):
        """tokens [n] of the sequences of tables, behind their first lens -> logits [n][vocab]; attend(layer, q, k, v)."""
        x = self.embed[tokens]
        for i, w in enumerate(self.layers):
            qkv = (x @ w["qkv"]).view(len(tokens), -1, self.d)
            v = qkv[:, self.hq + self.kvh:]
            q = cache.append(qkv[:, : self.hq], qkv[:, self.hq: self.hq + self.kvh], v, tables, lens, self.inv_freq, layer=i,
                             starts=starts, q_weight=w["wq"], k_weight=w["wk"], k_out=k_out)
            x = x + attend(i, q, k_out, v).reshape(x.shape) @ w["out"]
            x = x / x.float().square().mean(-1, keepdim=True).sqrt().to(BF)
        return x @ self.head


def run(samples=4, tokens=40, pages=0, prompt_len=200, page=32, seed=0):
    """([samples][tokens] sampled tokens, the prompt, the logits that the last of them was sampled from, the model); pages: of
    each sample and KV head in a step (0: all)."""
    if samples < 1 or tokens < 1 or prompt_len < 1 or pages < 0:
        raise ValueError("needs samples, tokens and a prompt, and pages >= 0")
    g = torch.Generator(device="cuda").manual_seed(seed)
    model = ToyModel(seed=seed)
    prompt = torch.randint(0, model.vocab, (prompt_len,), device="cuda", generator=g)
    # whole pages; what is left of the prompt, one token at least, every sample stores for itself
    shared = (prompt_len - 1) // page * page
    width = -(-(prompt_len + tokens) // page)
    own = width - shared // page
    cache = dc.PagedCache(len(model.layers), shared // page + samples * own, model.kvh, model.d, page_size=page, q_heads=model.hq)
    common = torch.arange(shared // page, dtype=torch.int32, device="cuda")
    mine = common.numel() + torch.arange(samples * own, dtype=torch.int32, device="cuda").view(samples, own)
    tables = torch.cat([common.expand(samples, -1), mine], 1).contiguous()

    # the shared part of the prompt once, then each sample's rest of it
    head, rest = prompt[:shared], prompt[shared:]
    if shared:
        zero = torch.zeros(1, dtype=torch.int32, device="cuda")
        keys = torch.empty((shared, model.kvh, model.d), dtype=BF, device="cuda")
        plan = dc.PromptPlan([shared], model.kvh, model.d, q_heads=model.hq)
        model.forward(head, cache, tables[:1].contiguous(), zero, lambda i, q, k, v: plan.attend(q, k, v), k_out=keys)
    prefixes = cache.share([samples], [shared])
    lens = torch.full((samples,), shared, dtype=torch.int32, device="cuda")

    def dense(i, q, k, v):
        return cache.attend(q, tables, lens + 1, layer=i, shared=prefixes)

    def sparse(i, q, k, v):
        # the newest page always, then the first one, then the one before the newest, as far as there is room
        selected = cache.select(q, tables, lens + 1, pages, layer=i, keep_first=min(1, pages - 1), keep_last=min(2, max(1, pages - 1)))
        return cache.attend(q, tables, lens + 1, layer=i, selected=selected)

    for t in rest.tolist():
        logits = model.forward(torch.full((samples,), t, device="cuda"), cache, tables, lens, dense)
        lens += 1

    token = torch.empty(samples, dtype=torch.long, device="cuda")
    noise = torch.empty((samples, model.vocab), device="cuda")
    state = {}

    def step():
        state["logits"] = model.forward(token, cache, tables, lens, sparse if pages else dense)
        lens.add_(1)
        token.copy_((state["logits"].float() + noise).argmax(-1))

    draw = lambda: -torch.log(-torch.log(torch.rand(noise.shape, device="cuda", generator=g).clamp(1e-9, 1 - 1e-7)))  # noqa: E731
    token.copy_((logits.float() + draw()).argmax(-1))
    out = [token.clone()]
    if tokens == 1:
        cache.check()
        return torch.stack(out, 1), prompt, logits, model
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # once outside of the capture: the libraries' own set-up
        before = token.clone(), lens.clone()
        noise.zero_()
        step()
        token.copy_(before[0])
        lens.copy_(before[1])
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        step()
    for _ in range(tokens - 1):
        noise.copy_(draw())
        graph.replay()
        out.append(token.clone())
    cache.check()
    return torch.stack(out, 1), prompt, state["logits"].clone(), model


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--samples", type=int, default=4)
    p.add_argument("--tokens", type=int, default=40)
    p.add_argument("--pages", type=int, default=0, help="pages of each sample and KV head in a step (0: all)")
    a = p.parse_args()
    if a.samples < 1 or a.tokens < 1 or a.pages < 0:
        p.error("--samples and --tokens must be at least 1, --pages at least 0")
    out = run(a.samples, a.tokens, a.pages)[0]
    for i, row in enumerate(out.tolist()):
        print(f"sample {i}: {row}")


if __name__ == "__main__":
    main()
