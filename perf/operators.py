"""The operators around the cache, as cases that can be timed: queries and keys normalised and
rotated, attention over packed prompts, and attention of drafted trees over a cache.

`own` picks the form that `run` takes: the framework's calls, or elementary torch operations in 32
bits. `listed` names the cases, `draw` gives another one of the same ranges, `prepare` makes a
case's inputs on the GPU from a seed, `run` is one pass, `work` its unavoidable bytes and
operations, `exact` the same outputs in 64 bits from the definitions.
"""

import math

import torch

own = False


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def _rotate(name, tokens, kvh, group, d, rot, dtype="bf16", norm=True, interleaved=False, first=0):
    return dict(name=name, kind="rotate", tokens=tokens, kvh=kvh, group=group, d=d, rot=rot, dtype=dtype, norm=norm,
                interleaved=interleaved, first=first)


def _prompt(name, q_lens, kvh, group, d, k_lens=None, dtype="bf16", causal=True):
    text = lambda v: " ".join(str(x) for x in v)  # noqa: E731
    return dict(name=name, kind="prompt", q_lens=text(q_lens), k_lens=text(k_lens or q_lens), kvh=kvh, group=group, d=d,
                dtype=dtype, causal=causal)


def _tree(name, layers, batch, kvh, group, d, n, nodes, shape="random"):
    return dict(name=name, kind="tree", layers=layers, batch=batch, kvh=kvh, group=group, d=d, n=n, nodes=nodes, shape=shape)


def listed():
    return [
        # one decode step of 8 sequences in one Mistral-7B-shaped layer: all latency
        _rotate("rotate_decode_8", 8, 8, 4, 128, 128, first=32768),
        # a prompt's layer: 8 sequences of 4096 tokens
        _rotate("rotate_prompt_32k", 32768, 8, 4, 128, 128),
        # a small model that rotates half of its dims, interleaved, without a norm, on an odd chunk
        _rotate("rotate_part_fp16", 1237, 2, 8, 64, 32, dtype="fp16", norm=False, interleaved=True, first=4091),
        # the smallest prompt: 512 tokens, 2 KV heads of 64 dims
        _prompt("prompt_tiny_512", [512], 2, 2, 64),
        # packed requests of ordinary, odd lengths in one layer, one of them a single token
        _prompt("prompt_packed_ragged", [1, 17, 130, 301, 512, 777, 1000, 1333, 2049, 2500], 8, 4, 128),
        # a 32K prompt, one layer
        _prompt("prompt_32k", [32768], 8, 4, 128),
        # a chunk of a prompt and a chat turn after long contexts, eight query heads per KV head, fp16
        _prompt("prompt_chunks_gqa8_fp16", [512, 100], 4, 8, 128, k_lens=[16384, 8292], dtype="fp16"),
        # single tokens against full caches of uneven lengths: 8 sequences up to 32K
        _prompt("prompt_single_tokens", [1] * 8, 8, 4, 128, k_lens=[32768, 30011, 24576, 16385, 12000, 8192, 4097, 1]),
        # the smallest tree: one layer, 2 KV heads of 64 dims, 128 tokens kept, 5 nodes
        _tree("tree_tiny", 1, 1, 2, 2, 64, 128, 5),
        # one layer of one sequence, 2048 of 8K kept, a chain of 4 drafted tokens
        _tree("tree_1layer_chain4", 1, 1, 8, 4, 128, 2048, 4, shape="chain"),
        # the benchmark's cache (32 layers, 8 sequences, 8192 kept), 16 nodes
        _tree("tree_seq8_8k_16", 32, 8, 8, 4, 128, 8192, 16),
        # a wide tree of 64 nodes with eight query heads per KV head over an odd length
        _tree("tree_gqa8_seq2_64", 32, 2, 4, 8, 128, 4097, 64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the same ranges, no dearer than the largest listed."""
    kind = rng.choice(["rotate", "prompt", "tree"])
    d = rng.choice([64, 128, 128])
    kvh, group = rng.choice([1, 2, 4, 8, 8]), rng.choice([1, 2, 4, 4, 8])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    if kind == "rotate":
        c = _rotate("", _log(rng, 1, 32768), kvh, group, d, rng.choice([d, d, d // 2]), dtype, rng.random() < 0.7,
                    rng.random() < 0.3, _log(rng, 1, 131072))
    elif kind == "prompt":
        while True:
            group = rng.choice([1, 2, 3, 4, 4, 5, 8])
            count = _log(rng, 1, 24)
            q = [_log(rng, 1, 8192) for _ in range(count)]
            more = rng.choice([0, 0, 1])
            k = [x + more * (_log(rng, 1, 16384) - 1) for x in q]
            if rng.random() < 0.25:
                k = [max(0, x + rng.randint(-3, 3)) for x in k]  # some rows see nothing
            causal = rng.random() < 0.85
            if sum(a * b for a, b in zip(q, k)) * kvh * group <= 1 << 33 and sum(k) <= 1 << 17 and sum(k) > 0:
                break
        c = _prompt("", q, kvh, group, d, k, dtype, causal)
    else:
        while True:
            c = _tree("", rng.choice([1, 1, 2, 4, 8, 16, 32]), _log(rng, 1, 16), kvh, group, d, _log(rng, 1, 32768),
                      _log(rng, 1, 128), rng.choice(["random", "random", "chain", "holes"]))
            rows = c["layers"] * c["batch"] * kvh
            if rows * c["n"] <= 1 << 23 and rows * c["n"] * c["nodes"] * group <= 1 << 31:
                break
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# Inputs: from the seed alone, on the GPU
# ---------------------------------------------------------------------------
_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _gen(seed, stream):
    return torch.Generator(device="cuda").manual_seed(seed * 16 + stream)


def _ints(text):
    return [int(x) for x in text.split()]


def _keys(shape, u, g, dtype):
    """Keys [..., tokens, d]: N(0, I), the first four scaled (sinks), 1% along the direction u (heavy hitters)."""
    x = torch.randn(shape, device="cuda", generator=g)
    x[..., :4, :] *= 2.0
    x += (torch.rand(shape[:-1] + (1,), device="cuda", generator=g) < 0.01) * (4.0 * u)
    return x.to(dtype)


def _parents(c, seed):
    """int32 [batch][nodes]: random trees, chains, or random trees with unused nodes (-2) among them."""
    g, b, T = _gen(seed, 5), c["batch"], c["nodes"]
    at = torch.arange(T, device="cuda")
    if c["shape"] == "chain":
        return (at - 1).to(torch.int32).expand(b, T).contiguous()
    p = (torch.rand((b, T), device="cuda", generator=g) * (at + 1)).to(torch.int32) - 1
    p = torch.minimum(p, at - 1).to(torch.int32)
    if c["shape"] == "holes":
        p[torch.rand((b, T), device="cuda", generator=g) < 0.3] = -2
    return p


def _inputs(c, seed):
    g, dt = _gen(seed, 1), _TYPES[c.get("dtype", "bf16")]
    kvh, G, d = c["kvh"], c["group"], c["d"]
    if c["kind"] == "rotate":
        T = c["tokens"]
        qkv = torch.randn((T, kvh * (G + 2), d), device="cuda", generator=g).to(dt)  # a fused projection's output
        w = [1 + 0.1 * torch.randn(d, device="cuda", generator=g) for _ in range(2)] if c["norm"] else [None, None]
        # packed sequences: positions rise from `first` and start again
        pos = (c["first"] + torch.arange(T, device="cuda") % 4096).to(torch.int32)
        f = (10000.0 ** (-torch.arange(0, c["rot"], 2, device="cuda", dtype=torch.float64) / c["rot"])).float()
        return dict(q=qkv[:, : kvh * G], k=qkv[:, kvh * G: kvh * (G + 1)], positions=pos, inv_freq=f, q_weight=w[0],
                    k_weight=w[1])
    if c["kind"] == "prompt":
        Tq, Tk = sum(_ints(c["q_lens"])), sum(_ints(c["k_lens"]))
        u = torch.randn((kvh, 1, d), device="cuda", generator=g)
        k = _keys((kvh, Tk, d), u, g, dt).transpose(0, 1).contiguous()
        v = torch.randn((Tk, kvh, d), device="cuda", generator=g).to(dt)
        q = torch.randn((Tq, kvh, G, d), device="cuda", generator=g) + 0.1 * u
        return dict(q=q.view(Tq, kvh * G, d).to(dt), k=k, v=v)
    L, b, n, T = c["layers"], c["batch"], c["n"], c["nodes"]
    u = torch.randn((L, b, kvh, 1, d), device="cuda", generator=g)
    k = torch.empty((L, b, kvh, n, d), dtype=dt, device="cuda")
    v = torch.empty_like(k)
    for layer in range(L):
        k[layer] = _keys((b, kvh, n, d), u[layer], g, dt)
        v[layer] = torch.randn((b, kvh, n, d), device="cuda", generator=g)
    q = torch.randn((L, b, T, kvh, G, d), device="cuda", generator=g) + 0.1 * u.view(L, b, 1, kvh, 1, d)
    kd, vd = (torch.randn((L, b, kvh, T, d), device="cuda", generator=g).to(dt) for _ in range(2))
    return dict(q=q.view(L, b, T, kvh * G, d).to(dt), k_draft=kd, v_draft=vd, parents=_parents(c, seed), k=k, v=v)


def prepare(case, seed):
    c = case
    s = dict(case=c, x=_inputs(c, seed))
    if own:
        from paper_2608_08878_gb300 import dc
        s["dc"] = dc
        if c["kind"] == "prompt":
            s["plan"] = dc.PromptPlan(_ints(c["q_lens"]), c["kvh"], c["d"], q_heads=c["kvh"] * c["group"],
                                      k_lens=_ints(c["k_lens"]), causal=c["causal"])
        if c["kind"] == "tree":
            s["cache"] = dc.DistillCache(c["layers"], c["kvh"], c["d"], c["n"] + c["nodes"], max(1, c["n"] - 1),
                                         batch=c["batch"], q_heads=c["kvh"] * c["group"])
            s["cache"].append(s["x"].pop("k"), s["x"].pop("v"))
    return s


def run(state):
    s = state
    c, x = s["case"], s["x"]
    if not own:
        return {"rotate": _plain_rotate, "prompt": _plain_prompt, "tree": _plain_tree}[c["kind"]](c, x, torch.float32)
    if c["kind"] == "rotate":
        return s["dc"].norm_rotate(x["q"], x["k"], x["positions"], x["inv_freq"], x["q_weight"], x["k_weight"],
                                   norm=c["norm"], interleaved=c["interleaved"])
    if c["kind"] == "prompt":
        return s["plan"].attend(x["q"], x["k"], x["v"], with_lse=True)
    return s["cache"].tree_attend(x["q"], x["k_draft"], x["v_draft"], x["parents"])


# ---------------------------------------------------------------------------
# The plain forms
# ---------------------------------------------------------------------------
EPS = 1e-6


def _plain_rotate(c, x, num):
    a = x["positions"].to(num)[:, None, None] * x["inv_freq"].to(num)
    cos, sin = torch.cos(a), torch.sin(a)

    def one(t, w):
        y = t.to(num)
        if c["norm"]:
            y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + EPS) * w.to(num)
        r, rest = y[..., : c["rot"]], y[..., c["rot"]:]
        if c["interleaved"]:
            p, q = r[..., 0::2], r[..., 1::2]
            r = torch.stack([p * cos - q * sin, q * cos + p * sin], -1).flatten(-2)
        else:
            p, q = r.chunk(2, -1)
            r = torch.cat([p * cos - q * sin, q * cos + p * sin], -1)
        return torch.cat([r, rest], -1).to(t.dtype)

    return one(x["q"], x["q_weight"]), one(x["k"], x["k_weight"])


def _softmax_sum(s, seen, v):
    """Scores s [..., r, keys], seen (broadcast to s) -> the weighted sum of v [..., keys, d] and log sum exp; 0 and
    -infinity where nothing is seen."""
    s = s.masked_fill(~seen, -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = torch.exp(s - m)
    l = p.sum(-1, keepdim=True)
    return p @ v / torch.where(l == 0, torch.ones_like(l), l), (m + torch.log(l)).squeeze(-1)


def _plain_prompt(c, x, num):
    kvh, G, d = c["kvh"], c["group"], c["d"]
    out = torch.zeros_like(x["q"])
    lse = torch.full(x["q"].shape[:2], -math.inf, dtype=num, device="cuda")
    q0 = k0 = 0
    for ql, kl in zip(_ints(c["q_lens"]), _ints(c["k_lens"])):
        k = x["k"][k0: k0 + kl].to(num).transpose(0, 1)
        v = x["v"][k0: k0 + kl].to(num).transpose(0, 1)
        rows = max(1, (1 << 28) // max(1, kvh * G * kl))  # blocks of queries: the scores of all at once need not fit
        for a in range(0, ql if kl else 0, rows):
            r = min(rows, ql - a)
            seen = torch.arange(kl, device="cuda") < kl
            if c["causal"]:
                seen = torch.arange(kl, device="cuda") <= torch.arange(a, a + r, device="cuda")[:, None] + (kl - ql)
            see = max(1, min(kl, a + r + kl - ql)) if c["causal"] else kl  # no query of the block sees further
            q = x["q"][q0 + a: q0 + a + r].to(num).view(r, kvh, G, d).permute(1, 2, 0, 3).reshape(kvh, G * r, d)
            s = (q @ k[:, :see].transpose(1, 2) / math.sqrt(d)).view(kvh, G, r, see)
            o, z = _softmax_sum(s, seen[..., :see].expand(r, see), v[:, None, :see])
            out[q0 + a: q0 + a + r] = o.permute(2, 0, 1, 3).reshape(r, kvh * G, d).to(out.dtype)
            lse[q0 + a: q0 + a + r] = z.permute(2, 0, 1).reshape(r, kvh * G)
        q0, k0 = q0 + ql, k0 + kl
    return out, lse


def _ancestors(parents, nodes):
    """[batch][nodes][nodes] truth values: column j is row i's node itself or one of its ancestors; no column for an unused node."""
    at = torch.arange(nodes, device="cuda")
    fine = (parents >= -1) & (parents < at)
    up = (parents[..., None] == at) & fine[..., None]
    reach = (up | torch.eye(nodes, dtype=torch.bool, device="cuda")).float()
    for _ in range(max(1, nodes - 1).bit_length()):  # paths of twice the length
        reach = (reach @ reach > 0).float()
    used = (reach @ ((parents == -1).float()[..., None]) > 0)
    return (reach > 0) & used


def _plain_tree(c, x, num):
    L, b, kvh, G, d, n, T = (c[k] for k in ("layers", "batch", "kvh", "group", "d", "n", "nodes"))
    anc = _ancestors(x["parents"], T)
    used = anc.any(-1, keepdim=True)
    seen = torch.cat([used.expand(b, T, n), anc], -1)[:, None, :, None].expand(b, kvh, T, G, n + T)
    out = torch.empty_like(x["q"])
    for layer in range(L):
        k = torch.cat([x["k"][layer], x["k_draft"][layer]], -2).to(num)
        v = torch.cat([x["v"][layer], x["v_draft"][layer]], -2).to(num)
        q = x["q"][layer].to(num).view(b, T, kvh, G, d).transpose(1, 2).reshape(b, kvh, T * G, d)
        s = q @ k.transpose(2, 3) / math.sqrt(d)
        o, _ = _softmax_sum(s, seen.reshape(b, kvh, T * G, n + T), v)
        out[layer] = o.view(b, kvh, T, G, d).transpose(1, 2).reshape(b, T, kvh * G, d).to(out.dtype)
    return out


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def _seen_pairs(c):
    """Query-key pairs of a prompt case, and keys that some query sees."""
    pairs = keys = 0
    for ql, kl in zip(_ints(c["q_lens"]), _ints(c["k_lens"])):
        if not c["causal"]:
            pairs, keys = pairs + ql * kl, keys + kl
            continue
        first = max(0, ql - kl)  # queries before it see nothing; query first sees first + kl - ql + 1 keys
        m, low = ql - first, first + kl - ql + 1
        pairs += m * low + m * (m - 1) // 2
        keys += kl if ql else 0
    return pairs, keys


def work(case):
    c = case
    kvh, G, d = c["kvh"], c["group"], c["d"]
    if c["kind"] == "rotate":
        values = c["tokens"] * kvh * (G + 1) * d
        return {"bytes": 4 * values + 4 * c["tokens"], "flops": (3 * c["norm"] + 3) * values}
    if c["kind"] == "prompt":
        pairs, keys = _seen_pairs(c)
        Tq = sum(_ints(c["q_lens"]))
        return {"bytes": 4 * Tq * kvh * G * d + 4 * keys * kvh * d + 4 * Tq * kvh * G, "flops": 4 * pairs * kvh * G * d}
    rows, T = c["layers"] * c["batch"] * c["kvh"], c["nodes"]
    return {"bytes": rows * (4 * d * (c["n"] + T) + 4 * T * G * d), "flops": 4 * d * rows * G * T * c["n"]}


# ---------------------------------------------------------------------------
# The same outputs in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def _attend64(q, k, v, seen):
    """Softmax attention in 64 bits: q [..., r, d], k, v [..., n, d], seen [..., r, n] -> output, log sum exp."""
    z = torch.einsum("...rd,...nd->...rn", q, k) * q.shape[-1] ** -0.5
    z = torch.where(seen, z, torch.full((), -math.inf, dtype=z.dtype, device=z.device))
    lse = torch.logsumexp(z, -1)
    w = torch.where(seen, torch.exp(z - torch.where(lse == -math.inf, 0.0, lse)[..., None]), 0.0)
    return torch.einsum("...rn,...nd->...rd", w, v), lse


def exact(case, seed):
    c, x = case, _inputs(case, seed)
    kvh, G, d = c["kvh"], c["group"], c["d"]
    if c["kind"] == "rotate":
        # each pair as a complex number, turned by its angle
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                           x["positions"].double()[:, None, None] * x["inv_freq"].double())
        outs = []
        for t, w in ((x["q"], x["q_weight"]), (x["k"], x["k_weight"])):
            y = t.double()
            if c["norm"]:
                y = y * w.double() * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS)
            h = c["rot"] // 2
            r = y[..., : c["rot"]].unflatten(-1, (h, 2) if c["interleaved"] else (2, h))
            r = r if c["interleaved"] else r.transpose(-1, -2)
            r = torch.view_as_real(torch.view_as_complex(r.contiguous()) * turn)
            r = (r if c["interleaved"] else r.transpose(-1, -2)).flatten(-2)
            outs.append(torch.cat([r, y[..., c["rot"]:]], -1))
        return tuple(outs)
    if c["kind"] == "prompt":
        if work(c)["flops"] > 1.2e13:
            return None
        outs, lses = [], []
        q0 = k0 = 0
        for ql, kl in zip(_ints(c["q_lens"]), _ints(c["k_lens"])):
            q = x["q"][q0: q0 + ql].double().view(ql, kvh, G, d)
            k, v = (x[t][k0: k0 + kl].double().transpose(0, 1)[:, None] for t in ("k", "v"))
            step = max(1, (1 << 27) // max(1, kvh * G * kl))
            for a in range(0, ql, step):
                t = torch.arange(a, min(ql, a + step), device="cuda")
                far = kl if not c["causal"] else max(0, min(kl, int(t[-1]) + kl - ql + 1))
                lim = t + (kl - ql) if c["causal"] else torch.full_like(t, kl)
                seen = torch.arange(far, device="cuda")[None] <= lim[:, None]
                o, z = _attend64(q[t].permute(1, 2, 0, 3), k[..., :far, :], v[..., :far, :], seen)
                outs.append(o.permute(2, 0, 1, 3).reshape(len(t), kvh * G, d))
                lses.append(z.permute(2, 0, 1).reshape(len(t), kvh * G))
            q0, k0 = q0 + ql, k0 + kl
        return torch.cat(outs), torch.cat(lses)
    L, b, T, n = c["layers"], c["batch"], c["nodes"], c["n"]
    up = x["parents"].tolist()
    seen = torch.zeros((b, T, n + T), dtype=torch.bool)
    for s in range(b):
        for i, p in enumerate(up[s]):
            if p == -1:
                seen[s, i, :n] = True
            elif 0 <= p < i:
                seen[s, i] = seen[s, p]
            seen[s, i, n + i] = p == -1 or (0 <= p < i and bool(seen[s, p].any()))
    seen = seen.cuda()[:, None, :, None].expand(b, kvh, T, G, n + T).reshape(b, kvh, T * G, n + T)
    out = torch.empty(x["q"].shape, dtype=torch.float64, device="cuda")
    for layer in range(L):
        for s in range(b):
            q = x["q"][layer, s].double().view(T, kvh, G, d).transpose(0, 1).reshape(kvh, T * G, d)
            k, v = (torch.cat([x[t][layer, s], x[t + "_draft"][layer, s]], 1).double() for t in ("k", "v"))
            out[layer, s] = _attend64(q, k, v, seen[s])[0].view(kvh, T, G, d).transpose(0, 1).reshape(T, kvh * G, d)
    return out
