"""Speculative decoding over a budgeted cache, on a toy model with random weights.

One forward pass of a prompt: queries and keys normalised and rotated (`dc.norm_rotate`), the prompt's own
attention (`dc.PromptPlan`), its keys and values appended to each layer's cache. Then rounds: continuations of
the last token that stood in the text before make a tree of drafts, one pass over the tree verifies them
(`DistillCache.tree_attend`), the longest path that the model itself would have taken is accepted and its keys
and values appended; the last accepted token goes through `DistillCache.step`, which scores the cache and
evicts down to the budget.

    python examples/draft_tree.py [--budget N] [--tokens N]
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_08878_gb300 import dc  # noqa: E402

BF = torch.bfloat16


class ToyModel:
    """layers of attention over a cache each, tied embeddings; one sequence."""

    def __init__(self, layers=2, kv_heads=2, group=4, d=64, vocab=256, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.kvh, self.hq, self.d, dim = kv_heads, kv_heads * group, d, kv_heads * group * d
        rand = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
        self.embed = rand(vocab, dim).to(BF)
        self.layers = [dict(qkv=(rand(dim, (self.hq + 2 * kv_heads) * d) / dim ** 0.5).to(BF),
                            out=(rand(dim, dim) / dim ** 0.5).to(BF),
                            wq=1 + 0.1 * rand(d), wk=1 + 0.1 * rand(d)) for _ in range(layers)]
        self.inv_freq = (10000.0 ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)).float()

    def project(self, layer, x, positions):
        """x [tokens][dim] -> q [tokens][hq][d], k, v [tokens][kvh][d], rotated to their positions."""
        qkv = (x @ layer["qkv"]).view(len(x), -1, self.d)
        q, k, v = qkv.split([self.hq, self.kvh, self.kvh], 1)
        q, k = dc.norm_rotate(q, k, positions, self.inv_freq, layer["wq"], layer["wk"])
        return q, k, v

    def forward(self, tokens, positions, attend):
        """Logits [tokens][vocab], with attend(layer number, q, k, v) -> [tokens][hq][d] for the attention."""
        x = self.embed[tokens]
        for i, layer in enumerate(self.layers):
            o = attend(i, *self.project(layer, x, positions))
            x = torch.nn.functional.rms_norm(x + o.reshape(x.shape) @ layer["out"], x.shape[-1:])
        return (x @ self.embed.T).float()


def draft(text, depth=4, width=2):
    """(tokens, parents) of a tree: node 0 is the text's last token, below it what followed that token where it
    stood before, at most `width` times and `depth` tokens each; paths that start alike share their nodes."""
    nodes, parents = [text[-1]], [-1]
    places = [i for i in range(len(text) - 2, -1, -1) if text[i] == text[-1]][:width]
    for p in places:
        at = 0
        for t in text[p + 1: p + 1 + depth]:
            same = [i for i in range(1, len(nodes)) if parents[i] == at and nodes[i] == t]
            if same:
                at = same[0]
            else:
                nodes.append(t)
                parents.append(at)
                at = len(nodes) - 1
    return nodes, parents


def generate(model, prompt, count, budget, depth=4, width=2):
    """count tokens after the prompt, greedily; returns them and the number of passes that it took."""
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    T = len(prompt)
    caches = [dc.DistillCache(1, model.kvh, model.d, max(T, budget) + count + 64, budget, q_heads=model.hq)
              for _ in model.layers]
    plan = dc.PromptPlan([T], model.kvh, model.d, q_heads=model.hq)
    rows = lambda t: t.transpose(0, 1).contiguous()[None, None]  # noqa: E731  [tokens][heads][d] as the cache has it

    def attend_prompt(i, q, k, v):
        caches[i].append(rows(k), rows(v))
        return plan.attend(q, k, v)

    logits = model.forward(torch.tensor(prompt, device="cuda"), ints(list(range(T))), attend_prompt)
    plan.check()
    text, passes = list(prompt) + [int(logits[-1].argmax())], 0
    while len(text) < T + count:
        nodes, parents = draft(text, depth, width)
        depths = []
        for p in parents:
            depths.append(0 if p < 0 else depths[p] + 1)
        kept, tree = [], ints([parents])

        def attend_tree(i, q, k, v):
            kept.append((q, k, v))
            return caches[i].tree_attend(q[None, None], rows(k), rows(v), tree)[0, 0]

        # (node 0 is the text's last token, which no cache holds yet)
        logits = model.forward(torch.tensor(nodes, device="cuda"), ints([len(text) - 1 + x for x in depths]), attend_tree)
        best = logits.argmax(-1).tolist()
        path = [0]
        while True:
            follow = [i for i in range(1, len(nodes)) if parents[i] == path[-1] and nodes[i] == best[path[-1]]]
            if not follow or len(text) + len(path) >= T + count:
                break
            path.append(follow[0])
        for cache, (q, k, v) in zip(caches, kept):
            if len(path) > 1:
                cache.append(rows(k[path[:-1]]), rows(v[path[:-1]]))
            cache.step(q[None, path[-1:]], k[None, path[-1:]], v[None, path[-1:]])
        text += [nodes[i] for i in path[1:]] + [best[path[-1]]]
        passes += 1
    for cache in caches:
        cache.sync()
    return text[T:], passes, [c.length()[0] for c in caches]


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--budget", type=int, default=96)
    ap.add_argument("--tokens", type=int, default=120)
    a = ap.parse_args(argv)
    model = ToyModel()
    prompt = torch.randint(0, 256, (200,), generator=torch.Generator().manual_seed(1)).tolist()
    tokens, passes, lengths = generate(model, prompt, a.tokens, a.budget)
    print(f"{len(tokens)} tokens in {passes} passes, {lengths} tokens cached per layer (budget {a.budget})")
    return tokens, passes, lengths


if __name__ == "__main__":
    main()
