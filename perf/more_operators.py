"""The operators of a step of speculative decoding over the paged KV cache, in plain form and as this library has them.

A sequence drafts a tree of tokens (a chain is the simplest one): node 0 is the last token that is known to stand, every other
node continues its parent.  All nodes run through the model as the sequence's new tokens of one step, and the longest path that
the model's own distributions accept is kept.  Five kinds of work:

  rope     cs_kv_append_rope: the step's Q, K and V out of a fused projection; Q and K normed for each head (RMS, optional) and
           rotated by their positions, K and V appended to the pages, Q written for the attention call
  qk       cs_qk_rope: the same norm and rotation alone, Q and K written as rows
  attend   cs_paged_attention_tree: attention of one layer, where a node sees the sequence's cached tokens and the nodes that its
           mask names (itself and its ancestors)
  verify   cs_spec_verify: drafts held against the target's probabilities with given random numbers, and the token that follows
           the last accepted one
  commit   cs_kv_tree_commit: keys and values of the accepted nodes move to the slots behind the cached tokens, all layers

The walk of `verify`, for one sequence: at node n (0 first) the children are tried in ascending order.  What is left of the
target's row, R, starts as p[n] with weight Z = 1.  Child i with token x is accepted if
  drafts drawn from rows q:   u[i] * q[n][x] * Z < R[x];   a refusal makes R = max(p[n] - c q[n], 0), c += Z (c = 0 at first), Z = sum R
  fixed guesses (no rows q):  u[i] * Z < R[x];             a refusal takes R[x] off Z and sets R[x] = 0
and the walk goes on at the child; where no child is accepted (or there is none) the next token is drawn from R: the first one at
which the running sum of R passes u' * sum R.  Where nothing is left of R it is p[n] that is drawn from.

A case is a dict of plain values; lengths, trees, page numbers and accepted paths follow from the case alone (`lengths` seeds
them), what the tensors hold follows from prepare()'s seed.
"""
import math
import random

import torch

own = False

PAGE = 16

#: Query heads, kv heads, head dim, layers of the model shapes.
MODELS = {
    "tiny": (4, 2, 64, 4),
    "llama8b": (32, 8, 128, 32),
    "qwen7b": (28, 4, 128, 28),
    "qwen14b": (40, 8, 128, 48),
    "llama70b": (64, 8, 128, 80),
}


def _step(name, kind, model, seqs=0, new=(1, 1), ctx=(0, 0), branch=0, chunks=0, chunk=(0, 0), prior=(0, 0), dtype="bf16", norm=False, rotary=128, interleaved=False,
          axes=1, lengths=1):
    c = {"name": name, "kind": kind, "model": model, "dtype": dtype, "seqs": seqs, "new_lo": new[0], "new_hi": new[1], "ctx_lo": ctx[0], "ctx_hi": ctx[1], "branch": branch,
         "lengths": lengths}
    if kind != "attend":
        c.update(chunks=chunks, chunk_lo=chunk[0], chunk_hi=chunk[1], prior_lo=prior[0], prior_hi=prior[1], norm=norm, rotary=rotary, interleaved=interleaved, axes=axes)
    return c


def _verify(name, seqs, new, branch, vocab, drawn, lengths=1):
    return {"name": name, "kind": "verify", "seqs": seqs, "new_lo": new[0], "new_hi": new[1], "branch": branch, "vocab": vocab, "drawn": drawn, "lengths": lengths}


def _commit(name, model, layers, seqs, new, ctx, branch, lengths=1):
    return {"name": name, "kind": "commit", "model": model, "layers": layers, "seqs": seqs, "new_lo": new[0], "new_hi": new[1], "ctx_lo": ctx[0], "ctx_hi": ctx[1], "branch": branch,
            "lengths": lengths}


def listed():
    return [
        # the smallest step: a few short requests, a token each
        _step("tiny_rope", "rope", "tiny", 4, (1, 1), (17, 100), rotary=64),
        # a large prefill step of a model with normed heads: ragged prompt chunks beside online decodes
        _step("llama8b_rope", "rope", "llama8b", 128, (1, 1), (512, 4096), chunks=6, chunk=(700, 2600), prior=(0, 4096), dtype="f16", norm=True),
        # drafts of a full batch, rotated in pairs of neighbours, half of each head
        _step("llama8b_qk", "qk", "llama8b", 64, (4, 6), (512, 4096), rotary=64, interleaved=True),
        # images of a few thousand tokens each, with positions in time, height and width
        _step("qwen7b_qk", "qk", "qwen7b", chunks=3, chunk=(1500, 4000), prior=(0, 500), dtype="f16", norm=True, axes=3),
        # the smallest trees: two short requests
        _step("tiny_attend", "attend", "tiny", 2, (5, 8), (17, 100), 2),
        # a full batch with a short chain of drafts for each request
        _step("llama8b_attend_chains", "attend", "llama8b", 64, (4, 6), (512, 4096)),
        # fewer requests, large trees, half precision
        _step("qwen7b_attend_trees", "attend", "qwen7b", 16, (24, 64), (1000, 8192), 6, dtype="f16"),
        # long contexts
        _step("llama70b_attend_trees", "attend", "llama70b", 32, (8, 32), (2048, 32768), 4),
        # a few requests with trees of the likeliest tokens
        _verify("verify_trees", 4, (12, 16), 4, 32000, False),
        # a full batch of chains, drawn from a draft model
        _verify("verify_chains", 128, (5, 6), 0, 128256, True),
        # one layer group of a small model
        _commit("tiny_commit", "tiny", 4, 2, (5, 8), (17, 100), 2),
        # a full batch of trees
        _commit("llama8b_commit", "llama8b", 32, 64, (16, 64), (16, 200), 6),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(("rope", "qk", "attend", "verify", "commit"), (3, 2, 6, 4, 2))[0]
    lengths = rng.randrange(1 << 20)
    while kind == "verify":
        most = _log(rng, 1, 32)
        c = _verify("", _log(rng, 1, 256), (max(1, most // rng.choice((1, 1, 2))), most), rng.choice((0, 0, 1, 3, 6)), rng.choice((1001, 32000, 50257, 128256, 151936, _log(rng, 1000, 200000))),
                    rng.random() < 0.5, lengths)
        del c["name"]
        if sum(_new(c)) * c["vocab"] <= 9.0e7 and work(c)["bytes"] <= 1.3e8:
            return c
    model = rng.choices(("tiny", "llama8b", "qwen7b", "qwen14b", "llama70b"), (1, 3, 3, 3, 3))[0]
    hq, hkv, d, most_layers = MODELS[model]
    dtype = "bf16" if rng.random() < 0.6 else "f16"
    while kind == "commit":
        most = _log(rng, 2, 64)
        c = _commit("", model, rng.randint(1, most_layers), _log(rng, 1, 64), (max(2, most // rng.choice((1, 2, 4))), most), (0, _log(rng, 1, 200)), rng.randint(1, 8), lengths)
        del c["name"]
        lengths += 1
        if work(c)["bytes"] > 0 and sum(_blocks(x + q) for x, q in _lengths(c)) * c["layers"] * 2 * hkv * PAGE * d * 2 <= 2.5e9:
            return c
    while kind == "attend":
        lo = _log(rng, 1, 8192)
        most = _log(rng, 1, 128)
        c = _step("", kind, model, _log(rng, 1, 64), (max(1, most // rng.choice((1, 1, 2, 4))), most), (lo, _log(rng, lo, 32768)), rng.choice((0, 1, 2, 4, 8)), dtype=dtype, lengths=lengths)
        del c["name"]
        seqs = _lengths(c)
        longest, new = max(x + q for x, q in seqs), max(q for _, q in seqs)
        if work(c)["bytes"] <= 2.1e9 and work(c)["flops"] <= 2.5e11 and len(seqs) * longest * hkv * d <= 1.1e9 and len(seqs) * longest * hq * new <= 2.1e9:
            return c
    while True:
        sides = rng.choice(("seqs", "chunks", "both"))
        most, long = _log(rng, 1, 32), _log(rng, 2, 4000)
        c = _step("", kind, model, 0 if sides == "chunks" else _log(rng, 1, 256), (max(1, most // rng.choice((1, 2))), most), (0, _log(rng, 1, 32768)), rng.choice((0, 2)),
                  0 if sides == "seqs" else rng.choice((1, 2, 3, 6)), (max(2, long // rng.choice((1, 3))), long), (0, rng.choice((0, _log(rng, 1, 4096)))), dtype, rng.random() < 0.5,
                  rng.choice((d, d, d // 2, d // 4)), rng.random() < 0.4, rng.choice((1, 1, 3)), lengths)
        del c["name"]
        if work(c)["bytes"] <= 2.3e8 and (kind == "qk" or sum(_blocks(x + q) for x, q in _lengths(c)) * 2 * hkv * PAGE * d * 2 <= 2.5e9):
            return c


# ---------------------------------------------------------------------------------- sizes

def _new(case):
    r = random.Random(case["lengths"])
    return [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])]


def _lengths(case):
    """(cached tokens, new tokens) of every sequence, the drafting ones first."""
    r = random.Random(case["lengths"] + 1)
    seqs = [(r.randint(case["ctx_lo"], case["ctx_hi"]), q) for q in _new(case)]
    return seqs + [(r.randint(case["prior_lo"], case["prior_hi"]), r.randint(case["chunk_lo"], case["chunk_hi"])) for _ in range(case.get("chunks", 0))]


def _trees(case):
    """The parents of every drafting sequence's nodes, -1 for node 0: one of the `branch` + 1 nodes before."""
    r = random.Random(case["lengths"] + 2)
    return [[-1] + [r.randint(max(0, i - 1 - case["branch"]), i - 1) for i in range(1, n)] for n in _new(case)]


def _depths(parents):
    depth = []
    for p in parents:
        depth.append(0 if p < 0 else depth[p] + 1)
    return depth


def _paths(case):
    """The accepted nodes of every sequence: down the tree from node 0, by chance as far as a leaf."""
    r = random.Random(case["lengths"] + 3)
    paths = []
    for parents in _trees(case):
        path = [0]
        while True:
            children = [i for i, p in enumerate(parents) if p == path[-1]]
            if not children or r.random() < 0.1:
                break
            path.append(r.choice(children))
        paths.append(path)
    return paths


def _blocks(n):
    return -(-n // PAGE)


def work(case):
    if case["kind"] == "verify":
        # a number for each node and sequence; the row of the node where the walk ends, and the drafts' one where they were drawn from rows
        nodes, rows = sum(_new(case)), case["seqs"]
        return {"bytes": nodes * (4 * 3 + 8) + rows * (8 + 4 * case["vocab"] * (2 if case["drawn"] else 1)), "flops": rows * case["vocab"] * (4 if case["drawn"] else 1)}
    hq, hkv, d, _ = MODELS[case["model"]]
    if case["kind"] == "commit":
        # K and V of the accepted nodes that do not lie where they belong, read and written; the paths and the pages' numbers
        moved = sum(n != k for path in _paths(case) for k, n in enumerate(path))
        return {"bytes": 2 * moved * case["layers"] * 2 * hkv * d * 2 + moved * 12, "flops": 0}
    tokens = sum(q for _, q in _lengths(case))
    if case["kind"] == "attend":
        nbytes = flops = 0
        for (c, q), parents in zip(_lengths(case), _trees(case)):
            # K, V and the page table read once, Q and a word of its mask read and the output written once
            nbytes += (c + q) * 2 * hkv * d * 2 + _blocks(c + q) * 4 + 2 * q * hq * d * 2 + 8 * q * -(-q // 64)
            flops += 4 * hq * d * (q * c + sum(_depths(parents)) + q)
        return {"bytes": nbytes, "flops": flops}
    # Q and K (and V) read and written, the positions and the frequencies read
    heads = hq + hkv * (2 if case["kind"] == "rope" else 1)
    return {"bytes": tokens * (2 * heads * d * 2 + 4 * case["axes"]) + case["rotary"] * 2, "flops": tokens * (hq + hkv) * d * (6 if case["norm"] else 3)}


# --------------------------------------------------------------------------------- inputs

def _tables(seqs, cpu):
    """Block tables over a pool without a page to spare, its pages shuffled."""
    need = [_blocks(c + q) for c, q in seqs]
    tables = torch.full((len(seqs), max(need)), -1, dtype=torch.int32)
    tables[torch.arange(max(need)) < torch.tensor(need)[:, None]] = torch.randperm(sum(need), generator=cpu).to(torch.int32)
    return tables, sum(need)


def _batch_arrays(seqs):
    ctx = torch.tensor([c for c, _ in seqs], dtype=torch.int32)
    cu = torch.zeros(len(seqs) + 1, dtype=torch.int32)
    cu[1:] = torch.cumsum(torch.tensor([q for _, q in seqs]), 0)
    return ctx, cu


def _masks(case):
    """int64 [T, words]: bit j of node i's words is set where j is i or an ancestor of it."""
    rows = []
    words = -(-max(_new(case)) // 64)
    for parents in _trees(case):
        seen = []
        for i, p in enumerate(parents):
            seen.append((seen[p] if p >= 0 else 0) | 1 << i)
        for m in seen:
            w = [m >> 64 * k & (1 << 64) - 1 for k in range(words)]
            rows.append([x - (1 << 64) if x >> 63 else x for x in w])
    return torch.tensor(rows, dtype=torch.int64)


def _prepare_step(case, seed):
    hq, hkv, d, _ = MODELS[case["model"]]
    cpu = torch.Generator().manual_seed(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = torch.float16 if case["dtype"] == "f16" else torch.bfloat16
    kind, seqs = case["kind"], _lengths(case)
    tables, pages = _tables(seqs, cpu)
    ctx, cu = _batch_arrays(seqs)
    total = int(cu[-1])
    s = {"kind": kind, "hq": hq, "hkv": hkv, "d": d, "dtype": dtype, "tables": tables.cuda(), "ctx": ctx.cuda(), "cu": cu.cuda(), "scale": 1 / math.sqrt(d),
         "longest": max(c + q for c, q in seqs), "most_new": max(q for _, q in seqs)}
    if kind != "qk":
        pool = torch.empty((1, pages, 2, hkv, PAGE * d), dtype=dtype, device="cuda").normal_(generator=gen)
        s["pool"] = pool
    if kind == "attend":
        s["q"] = torch.randn((total, hq, d), generator=gen, device="cuda", dtype=dtype)
        s["out"] = torch.empty_like(s["q"])
        s["mask"] = _masks(case).cuda()
    else:
        # what the projection wrote, its heads of several sizes
        row = torch.randn((total, hq + 2 * hkv, d), generator=gen, device="cuda") * torch.exp2(torch.randn((1, hq + 2 * hkv, 1), generator=gen, device="cuda"))
        row = row.to(dtype)
        s["q"], s["k"], s["v"] = row[:, :hq], row[:, hq:hq + hkv], row[:, hq + hkv:]
        s["q_out"] = torch.empty((total, hq, d), dtype=dtype, device="cuda")
        s["k_out"] = torch.empty((total, hkv, d), dtype=dtype, device="cuda")
        s["q_norm"], s["k_norm"] = ((1 + torch.randn(d, generator=gen, device="cuda") / 4).to(dtype) if case["norm"] else None for _ in range(2))
        pairs = case["rotary"] // 2
        s["rotary"], s["interleaved"], s["eps"] = case["rotary"], case["interleaved"], 1e-6
        s["freq"] = torch.pow(torch.tensor(500000.0, dtype=torch.float64), -torch.arange(pairs, dtype=torch.float64) / pairs).float().cuda()
        # a node stands at its depth behind the cached tokens; an image's token at a time, a height and a width
        first = torch.tensor([c for c, q in seqs for _ in range(q)])
        if case["axes"] == 1:
            at = torch.tensor([x for t in _trees(case) for x in _depths(t)] + [x for _, q in seqs[case["seqs"]:] for x in range(q)])
            s["axis_pairs"] = None
            s["positions"] = (first + at).to(torch.int32).cuda()[None]
        else:
            at = torch.tensor([x for _, q in seqs for x in range(q)])
            s["axis_pairs"] = [pairs - 2 * (3 * pairs // 8), 3 * pairs // 8, 3 * pairs // 8]
            s["positions"] = torch.stack([first + at // 1024, first + at // 32 % 32, first + at % 32]).to(torch.int32).cuda()
    if own:
        from paper_2410_01228_amd import binding as cs
        if kind == "qk":
            s["rope"] = cs.Rope(s["freq"], s["rotary"], s["positions"], s["axis_pairs"], s["interleaved"], s["q_norm"], s["k_norm"], s["eps"])
            return s
        s["batch"] = cs.Batch(tables, ctx, cu)
        s["handle"] = cs.Pool(s["pool"], 1, pages, hkv, d)
        if kind == "attend":
            s["workspace"] = cs.workspace_for_tree(s["batch"], hq, hkv, d)
        else:
            s["rope"] = cs.Rope(s["freq"], s["rotary"], s["positions"], s["axis_pairs"], s["interleaved"], s["q_norm"], s["k_norm"], s["eps"])
    return s


def _prepare_verify(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    trees, vocab = _trees(case), case["vocab"]
    cu = torch.zeros(len(trees) + 1, dtype=torch.int32)
    cu[1:] = torch.cumsum(torch.tensor([len(t) for t in trees]), 0)
    total = int(cu[-1])
    parents = torch.tensor([p for t in trees for p in t], dtype=torch.int32)
    # the row that a node was drafted from, and how many of its siblings come before it
    source = torch.tensor([int(cu[i]) + max(p, 0) for i, t in enumerate(trees) for p in t]).cuda()
    rank = torch.tensor([t[:j].count(p) for t in trees for j, p in enumerate(t)]).cuda()
    # the target's logits, and a draft model's that are near them
    x = torch.randn((total, vocab), generator=gen, device="cuda") * 3
    p = torch.softmax(x, -1)
    x += torch.randn((total, vocab), generator=gen, device="cuda")
    q = torch.softmax(x, -1)
    if case["drawn"]:
        tokens = torch.empty(total, dtype=torch.int64, device="cuda")
        for part in torch.arange(total).split(256):
            race = torch.empty((len(part), vocab), device="cuda").exponential_(generator=gen)
            tokens[part.cuda()] = (q[source[part.cuda()]] / race).argmax(-1)
    else:
        tokens = q.topk(min(vocab, int(rank.max()) + 1), -1).indices[source, rank]
        q = None
    s = {"kind": "verify", "seqs": len(trees), "most_new": max(len(t) for t in trees), "ranks": int(rank.max()) + 1, "cu": cu.cuda(), "tokens": tokens.to(torch.int32), "parents": parents.cuda(),
         "p": p, "q": q, "u": torch.rand(total, generator=gen, device="cuda"), "u_next": torch.rand(len(trees), generator=gen, device="cuda"),
         "out_tokens": torch.empty(total, dtype=torch.int32, device="cuda"), "path": torch.empty(total, dtype=torch.int32, device="cuda"),
         "count": torch.empty(len(trees), dtype=torch.int32, device="cuda")}
    if own:
        from paper_2410_01228_amd import binding as cs
        s["batch"] = cs.Batch(torch.zeros((len(trees), _blocks(max(len(t) for t in trees))), dtype=torch.int32), torch.zeros(len(trees), dtype=torch.int32), cu)
        s["workspace"] = cs.workspace_for_verify(s["batch"], vocab)
    return s


def _prepare_commit(case, seed):
    _, hkv, d, _ = MODELS[case["model"]]
    cpu = torch.Generator().manual_seed(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    seqs = _lengths(case)
    tables, pages = _tables(seqs, cpu)
    ctx, cu = _batch_arrays(seqs)
    path = torch.full((int(cu[-1]),), -1, dtype=torch.int32)
    for t0, nodes in zip(cu.tolist(), _paths(case)):
        path[t0:t0 + len(nodes)] = torch.tensor(nodes, dtype=torch.int32)
    pool = torch.empty((case["layers"], pages, 2, hkv, PAGE * d), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    s = {"kind": "commit", "hkv": hkv, "d": d, "layers": case["layers"], "pages": pages, "pool": pool, "tables": tables.cuda(), "ctx": ctx.cuda(), "cu": cu.cuda(), "path": path.cuda(),
         "count": torch.tensor([len(p) for p in _paths(case)], dtype=torch.int32).cuda()}
    if own:
        from paper_2410_01228_amd import binding as cs
        s["batch"] = cs.Batch(tables, ctx, cu)
        s["handle"] = cs.Pool(pool, case["layers"], pages, hkv, d)
    return s


def prepare(case, seed):
    return {"verify": _prepare_verify, "commit": _prepare_commit}.get(case["kind"], _prepare_step)(case, seed)


# ------------------------------------------------------------------------------ plain forms

def _views(pool, hkv, d):
    """K [layer, page, kv head, feature / 8, token, feature % 8] and V [layer, page, kv head, feature / 16, token / 8, feature % 16, token % 8] of a pool."""
    lead = pool.shape[:2]
    return pool[:, :, 0].view(*lead, hkv, d // 8, PAGE, 8), pool[:, :, 1].view(*lead, hkv, d // 16, 2, 16, 8)


def _where(s, total):
    """The sequence of each of the step's tokens, and its number in it."""
    token = torch.arange(total, device="cuda")
    cu = s["cu"].long()
    seq = torch.searchsorted(cu[1:], token, right=True)
    return seq, token - cu[seq]


def _plain_rotated(s, x, norm):
    """x [T, heads, D] normed and rotated, float32."""
    y = x.float()
    if norm is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + s["eps"]) * norm.float()
    pairs = s["rotary"] // 2
    at = s["positions"].double()
    if s["axis_pairs"] is not None:
        axis = torch.repeat_interleave(torch.arange(3, device="cuda"), torch.tensor(s["axis_pairs"], device="cuda"), output_size=pairs)
        angle = at[axis].T * s["freq"].double()
    else:
        angle = at[0][:, None] * s["freq"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    turned = y[..., :2 * pairs]
    if s["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = turned[..., :pairs], turned[..., pairs:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, y[..., 2 * pairs:]], -1)


def _plain_rope(s):
    hkv, d, dtype = s["hkv"], s["d"], s["dtype"]
    total = s["q"].shape[0]
    s["q_out"].copy_(_plain_rotated(s, s["q"], s["q_norm"]))
    k_new = _plain_rotated(s, s["k"], s["k_norm"]).to(dtype)
    if s["kind"] == "qk":
        s["k_out"].copy_(k_new)
        return {"q": s["q_out"], "k": s["k_out"]}
    seq, i = _where(s, total)
    pos = s["ctx"].long()[seq] + i
    page, slot = s["tables"].long()[seq, pos // PAGE], pos % PAGE
    k, v = _views(s["pool"], hkv, d)
    k[0, page, :, :, slot] = k_new.view(total, hkv, d // 8, 8)
    v[0, page, :, :, slot // 8, :, slot % 8] = s["v"].reshape(total, hkv, d // 16, 16)
    return {"q": s["q_out"], "pool": s["pool"]}


def _plain_attend(s):
    hq, hkv, d, n, most = s["hq"], s["hkv"], s["d"], s["tables"].shape[0], s["most_new"]
    ctx, cu, out = s["ctx"].long(), s["cu"].long(), s["out"]
    pages = s["tables"].long().clamp_min(0)
    k, v = _views(s["pool"], hkv, d)
    k = k[0, pages].float().permute(0, 2, 1, 4, 3, 5).reshape(n, hkv, -1, d)             # [n, Hkv, keys, D]
    v = v[0, pages].float().permute(0, 2, 1, 4, 6, 3, 5).reshape(n, hkv, -1, d)
    new = torch.arange(most, device="cuda")
    token = (cu[:-1, None] + new).clamp_max(s["q"].shape[0] - 1)
    q = s["q"][token].float().view(n, most, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, -1, d)
    key = torch.arange(k.shape[2], device="cuda")
    node = key - ctx[:, None]                                                             # [n, keys]
    there = node < (cu[1:] - cu[:-1])[:, None]
    v = torch.where(there[:, None, :, None], v, torch.zeros((), device="cuda"))
    bit = node.clamp(0, 64 * s["mask"].shape[1] - 1)
    word = s["mask"][token].gather(2, (bit // 64)[:, None].expand(-1, most, -1))
    seen = ((word >> (bit % 64)[:, None]) & 1).bool() | (node < 0)[:, None]
    seen &= there[:, None]                                                                # [n, new, keys]
    x = torch.matmul(q, k.transpose(2, 3)).view(n, hkv, hq // hkv, most, -1).mul_(s["scale"])
    x.masked_fill_(~seen[:, None, None], -math.inf)
    x -= x.amax(-1, keepdim=True).clamp_min(-3e38)
    x.exp_()
    total = x.sum(-1, keepdim=True)
    y = torch.matmul(x.view(n, hkv, -1, x.shape[-1]), v).view(n, hkv, hq // hkv, most, d) / torch.where(total > 0, total, 1.0)
    mine = new < (cu[1:] - cu[:-1])[:, None]
    out[token[mine]] = y.permute(0, 3, 1, 2, 4).reshape(n, most, hq, d)[mine].to(out.dtype)
    return out


def _plain_verify(s):
    n, most, drawn = s["seqs"], s["most_new"], s["q"] is not None
    cu = s["cu"].long()
    total = s["tokens"].shape[0]
    node = torch.arange(most, device="cuda")
    there = node < (cu[1:] - cu[:-1])[:, None]                                            # [n, nodes]
    token = (cu[:-1, None] + node).clamp_max(total - 1)
    x = s["tokens"].long()[token]
    parent = torch.where(there, s["parents"].long()[token], -1)
    row = (cu[:-1, None] + parent).clamp(0, total - 1)                                    # of what a node was drafted from
    u = s["u"].double()[token]
    px = s["p"][row, x].double()
    before = (parent[:, :, None] == parent[:, None]) & (parent >= 0)[:, :, None] & (node < node[:, None])     # [n, node, earlier sibling]
    rank = before.sum(-1)
    if drawn:
        # Z and c before each of a row's children
        c, z = [torch.zeros(total, dtype=torch.float64, device="cuda")], [torch.ones(total, dtype=torch.float64, device="cuda")]
        for _ in range(1, s["ranks"]):
            c.append(c[-1] + z[-1])
            z.append((s["p"].double() - c[-1][:, None] * s["q"].double()).clamp_min(0).sum(-1))
        c.append(c[-1] + z[-1])
        c, z = torch.stack(c, -1), torch.stack(z, -1)
        qx = s["q"][row, x].double()
        passed = u * qx * z[row, rank.clamp_max(s["ranks"] - 1)] < (px - c[row, rank.clamp_max(s["ranks"] - 1)] * qx).clamp_min(0)
    else:
        again = (before & (x[:, :, None] == x[:, None])).any(-1)
        gone = torch.where(again, 0.0, px)                                                # what its refusal takes off Z
        z = 1 - torch.matmul(before.double(), gone[..., None])[..., 0]
        passed = u * z < gone
    passed &= parent >= 0
    passed &= ~(before & passed[:, None]).any(-1)                                         # the first of its siblings
    passed |= (node == 0) & there
    # a node is kept if it and all of its ancestors have passed
    up = torch.where(parent < 0, node, parent)
    kept, jump = passed, up
    for _ in range(max(1, (most - 1).bit_length())):
        kept = kept & kept.gather(1, jump)
        jump = jump.gather(1, jump)
    count = kept.sum(-1)
    place = kept.cumsum(-1) - 1
    path = torch.full((n, most + 1), -1, dtype=torch.long, device="cuda").scatter_(1, torch.where(kept, place, most), node.expand(n, -1))[:, :most]
    last = path.gather(1, (count - 1).clamp_min(0)[:, None])
    end = (cu[:-1, None] + last)[:, 0].clamp(0, total - 1)
    p = s["p"][end].double()
    mine = parent == last                                                                 # its children, all refused
    if drawn:
        at = mine.sum(-1)
        left = (p - c[end, at][:, None] * s["q"][end].double()).clamp_min(0)
    else:
        left = torch.cat([p, p[:, :1]], 1).scatter_(1, torch.where(mine, x, p.shape[1]), 0.0)[:, :-1]
    left = torch.where(left.sum(-1, keepdim=True) > 0, left, p)
    running = left.cumsum(-1)
    drawn_at = (running <= s["u_next"].double()[:, None] * running[:, -1:]).sum(-1)
    final = left.shape[1] - 1 - (left.flip(-1) > 0).to(torch.int8).argmax(-1)              # for sums that never pass: the last with a weight
    next_ = torch.where(running[:, -1] > 0, torch.minimum(drawn_at, final), -1)
    kept_tokens = torch.where(node + 1 < count[:, None], x.gather(1, torch.cat([path[:, 1:], path[:, :1]], 1).clamp_min(0)), -1)
    kept_tokens.scatter_(1, (count - 1).clamp_min(0)[:, None], next_[:, None])
    s["count"].copy_(count)
    s["path"][token[there]] = path[there].to(torch.int32)
    s["out_tokens"][token[there]] = kept_tokens[there].to(torch.int32)
    return {"tokens": s["out_tokens"], "path": s["path"], "count": s["count"]}


def _plain_commit(s):
    total = s["path"].shape[0]
    seq, i = _where(s, total)
    tables, ctx = s["tables"].long(), s["ctx"].long()
    to = ctx[seq] + i
    of = ctx[seq] + torch.where(i < s["count"].long()[seq], s["path"].long(), i)          # the others stay where they are
    dp, dt, sp, st = tables[seq, to // PAGE], to % PAGE, tables[seq, of // PAGE], of % PAGE
    k, v = _views(s["pool"], s["hkv"], s["d"])
    k[:, dp, :, :, dt] = k[:, sp, :, :, st]
    v[:, dp, :, :, dt // 8, :, dt % 8] = v[:, sp, :, :, st // 8, :, st % 8]
    return s["pool"].view(torch.int32)


def run(state):
    s, kind = state, state["kind"]
    if not own:
        if kind in ("rope", "qk"):
            return _plain_rope(s)
        if kind == "attend":
            return _plain_attend(s)
        return _plain_verify(s) if kind == "verify" else _plain_commit(s)
    from paper_2410_01228_amd import binding as cs
    half = kind in ("rope", "qk", "attend") and s["dtype"] == torch.float16
    if kind == "rope":
        append = cs.cs_kv_append_rope_f16 if half else cs.cs_kv_append_rope
        append(s["handle"], 0, s["batch"], s["rope"], s["q"], s["k"], s["v"], s["q_out"])
        return {"q": s["q_out"], "pool": s["pool"]}
    if kind == "qk":
        rotate = cs.cs_qk_rope_f16 if half else cs.cs_qk_rope
        rotate(s["rope"], s["q"], s["k"], s["q_out"], s["k_out"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if kind == "attend":
        attend = cs.cs_paged_attention_tree_f16 if half else cs.cs_paged_attention_tree
        attend(s["handle"], 0, s["batch"], s["q"], s["out"], s["hq"], s["scale"], s["mask"], s["workspace"])
        return s["out"]
    if kind == "verify":
        cs.cs_spec_verify(s["batch"], s["tokens"], s["parents"], s["p"], s["q"], s["u"], s["u_next"], s["out_tokens"], s["path"], s["count"], s["workspace"])
        return {"tokens": s["out_tokens"], "path": s["path"], "count": s["count"]}
    cs.cs_kv_tree_commit(s["handle"], 0, s["layers"], s["batch"], s["path"], s["count"])
    return s["pool"].view(torch.int32)


# -------------------------------------------------------------------------- 64-bit definition

def _exact_rows(case, s, x, norm):
    """x [T, heads, D]: y = x / sqrt(mean x^2 + eps) * norm, then each pair (a, b) as the complex number (a + ib) e^(i angle)."""
    y = x.double()
    if norm is not None:
        y = y / torch.sqrt(torch.square(y).sum(-1, keepdim=True) / y.shape[-1] + s["eps"]) * norm.double()
    pairs = case["rotary"] // 2
    i = torch.arange(pairs, device="cuda")
    first, second = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + pairs)
    axis = torch.zeros_like(i)
    if case["axes"] == 3:
        axis += (i >= s["axis_pairs"][0]).long() + (i >= s["axis_pairs"][0] + s["axis_pairs"][1]).long()
    angle = s["positions"].double().index_select(0, axis).transpose(0, 1) * s["freq"].double()
    turned = torch.complex(y[..., first], y[..., second]) * torch.polar(torch.ones_like(angle), angle)[:, None]
    y = y.clone()
    y[..., first], y[..., second] = turned.real, turned.imag
    return y


def _exact_rope(case, s):
    hkv, d = s["hkv"], s["d"]
    q, k_new = _exact_rows(case, s, s["q"], s["q_norm"]), _exact_rows(case, s, s["k"], s["k_norm"])
    if case["kind"] == "qk":
        return {"q": q, "k": k_new}
    pool = s["pool"].double()
    f = torch.arange(d, device="cuda")
    head = torch.arange(hkv, device="cuda")[:, None]
    t = torch.tensor([(row[(c + j) // PAGE], (c + j) % PAGE) for row, (c, n) in zip(s["tables"].tolist(), _lengths(case)) for j in range(n)], device="cuda")
    page, slot = t[:, 0, None, None], t[:, 1, None, None]
    pool[0, page, 0, head, (f // 8 * PAGE + slot) * 8 + f % 8] = k_new
    pool[0, page, 1, head, ((f // 16 * 2 + slot // 8) * 16 + f % 16) * 8 + slot % 8] = s["v"].double()
    return {"q": q, "pool": pool}


def _exact_attend(case, s):
    hq, hkv, d = s["hq"], s["hkv"], s["d"]
    group = hq // hkv
    f, t = torch.arange(d, device="cuda"), torch.arange(PAGE, device="cuda")[:, None]
    where = ((f // 8 * PAGE + t) * 8 + f % 8, ((f // 16 * 2 + t // 8) * 16 + f % 16) * 8 + t % 8)
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    t0 = 0
    for i, ((c, n), parents) in enumerate(zip(_lengths(case), _trees(case))):
        raw = s["pool"][0, s["tables"][i, :_blocks(c + n)].long()]
        hidden = torch.ones((n, c + n), dtype=torch.bool)
        hidden[:, :c] = False
        for j, p in enumerate(parents):
            if p >= 0:
                hidden[j, c:] = hidden[p, c:]
            hidden[j, c + j] = False
        hidden = hidden.cuda()
        for g in range(hkv):
            k, v = (raw[:, kv, g][:, where[kv]].double().reshape(-1, d)[:c + n] for kv in (0, 1))
            x = torch.matmul(s["q"][t0:t0 + n, g * group:(g + 1) * group].double().transpose(0, 1), k.T) / math.sqrt(d)
            out[t0:t0 + n, g * group:(g + 1) * group] = torch.matmul(torch.softmax(x.masked_fill(hidden, -math.inf), -1), v).transpose(0, 1)
        t0 += n
    return out


def _exact_verify(case, s):
    """The walk, node by node."""
    tokens, path, count = [], [], []
    all_x, all_u, u_next = s["tokens"].tolist(), s["u"].double().tolist(), s["u_next"].double().tolist()
    t0 = 0
    for i, parents in enumerate(_trees(case)):
        at, walked = 0, [0]
        while True:
            p = s["p"][t0 + at].double()
            q = s["q"][t0 + at].double() if case["drawn"] else None
            left, z, c, went = p.clone(), 1.0, 0.0, None
            for j in (j for j, parent in enumerate(parents) if parent == at):
                x, u = all_x[t0 + j], all_u[t0 + j]
                r = float(left[x])
                if (u * float(q[x]) if case["drawn"] else u) * z < r:
                    went = j
                    break
                if case["drawn"]:
                    c += z
                    left = torch.clamp(p - c * q, min=0)
                    z = float(left.sum())
                else:
                    left[x] = 0
                    z -= r
            if went is None:
                break
            at = went
            walked.append(at)
        if not bool((left > 0).any()):
            left = p
        running = torch.cumsum(left, 0)
        passed = (running > u_next[i] * running[-1]).nonzero()
        some = (left > 0).nonzero()
        next_ = int(passed[0]) if len(passed) else int(some[-1]) if len(some) else -1
        row = [all_x[t0 + j] for j in walked[1:]] + [next_]
        tokens += row + [-1] * (len(parents) - len(row))
        path += walked + [-1] * (len(parents) - len(walked))
        count.append(len(walked))
        t0 += len(parents)
    return {"tokens": torch.tensor(tokens, dtype=torch.int32), "path": torch.tensor(path, dtype=torch.int32), "count": torch.tensor(count, dtype=torch.int32)}


def exact(case, seed):
    if case["kind"] == "commit":
        return None                                      # bytes that move: nothing is computed
    s = prepare(case, seed)
    return {"attend": _exact_attend, "verify": _exact_verify}.get(case["kind"], _exact_rope)(case, s)
