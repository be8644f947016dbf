"""The operators of the 8-bit KV cache and of its pages, in plain form and as this library has them.

Five kinds of work on pools of 16-token pages:

  append   cs_kv8_append: a step's new K/V rows rounded to 8 bits (e4m3), with one power-of-two scale
           for each (page, K or V, kv head) block of 16 tokens
  attend   cs_paged_attention_mixed_kv8: paged attention of one layer over such a pool, decode tokens
           and prefill chunks in one call
  copy     cs_kv_pages_copy: whole pages from one list of ids to another, all layers
  fork     a step of parallel sampling or beam search: cs_kv_pages_free drops the losing sequences,
           cs_kv_pages_fork starts new ones that share their parent's full pages
  compact  cs_kv_pages_compact: the pages in use move to the front of the pool

An 8-bit page is, in bytes, [K, V][kv head][16 * D] codes, then [K, V][kv head] scales (float32); token t
and feature d of a block are code
  K:  ((d / 16) * 16 + t) * 16 + d % 16
  V:  (((d / 64) * 4 + t / 4) * 16 + d % 16) * 16 + ((d / 16) % 4) * 4 + t % 4
and stand for code * scale.

A case is a dict of plain values; lengths and page numbers follow from the case alone (`lengths` seeds
them), what the tensors hold follows from prepare()'s seed.
"""
import math
import random

import torch

own = False

PAGE = 16
FP8 = torch.float8_e4m3fn
FP8_MAX = 448.0
#: Scales are powers of two, 2**-100 at least.
LOWEST_EXPONENT = -100
#: What half precision can hold of the values that 8 bits can: 2**16 is too much.
F16_MOST = 61440.0

#: Query heads, kv heads, head dim, layers of the model shapes.
MODELS = {
    "tiny": (4, 2, 64, 4),
    "llama8b": (32, 8, 128, 32),
    "qwen7b": (28, 4, 128, 28),
    "qwen14b": (40, 8, 128, 48),
    "llama70b": (64, 8, 128, 80),
}


def _step(name, kind, model, decodes=0, ctx=(0, 0), chunks=0, chunk=(0, 0), prior=(0, 0), dtype="bf16", lengths=1):
    return {"name": name, "kind": kind, "model": model, "dtype": dtype, "decodes": decodes, "ctx_lo": ctx[0], "ctx_hi": ctx[1],
            "chunks": chunks, "chunk_lo": chunk[0], "chunk_hi": chunk[1], "prior_lo": prior[0], "prior_hi": prior[1], "lengths": lengths}


def _pages(name, kind, model, layers, bits, lengths=1, **more):
    return {"name": name, "kind": kind, "model": model, "layers": layers, "bits": bits, "lengths": lengths, **more}


def listed():
    return [
        # the smallest step: a few short requests
        _step("tiny_append", "append", "tiny", 4, (17, 100), 2, (32, 32), (0, 48)),
        # a large prefill step: ragged prompt chunks on prior context that ends inside pages, beside online decodes
        _step("llama8b_append", "append", "llama8b", 128, (512, 4096), 6, (700, 2600), (0, 4096), dtype="f16"),
        # a quiet moment online: a handful of chat requests decode
        _step("llama8b_attend_few", "attend", "llama8b", 8, (128, 2048)),
        # a full decode batch, half precision
        _step("qwen14b_attend_decode", "attend", "qwen14b", 256, (512, 4096), dtype="f16"),
        # offline only: ragged prompt chunks fill the token budget
        _step("llama8b_attend_prefill", "attend", "llama8b", chunks=3, chunk=(300, 1200), prior=(0, 8192)),
        # co-serving with long contexts: online decodes and one offline chunk far into its prompt
        _step("llama70b_attend_mixed", "attend", "llama70b", 128, (2048, 32768), 1, (1024, 1024), (30720, 30720)),
        # one request's pages duplicated, 16-bit pool
        _pages("tiny_copy", "copy", "tiny", 4, 16, count=5),
        # offline requests' pages moved between allocations
        _pages("qwen14b_copy", "copy", "qwen14b", 48, 8, count=1152),
        # four samples of one prompt
        _pages("llama8b_fork", "fork", "llama8b", 32, 8, parents=1, children=4, len_lo=300, len_hi=1500),
        # beam search over a batch
        _pages("llama70b_fork", "fork", "llama70b", 80, 8, parents=64, children=8, len_lo=100, len_hi=2000),
        # a small pool after a few requests have left
        _pages("tiny_compact", "compact", "tiny", 4, 16, rows=9, prefix=2, len_lo=40, len_hi=300, spare=40, moves=21),
        # a fragmented pool, packed so that its tail can be given back
        _pages("qwen7b_compact", "compact", "qwen7b", 28, 8, rows=96, prefix=16, len_lo=500, len_hi=4000, spare=6000, moves=3100),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(("append", "attend", "copy", "fork", "compact"), (3, 7, 2, 2, 2))[0]
    model = rng.choices(("tiny", "llama8b", "qwen7b", "qwen14b", "llama70b"), (1, 3, 3, 3, 3))[0]
    lengths = rng.randrange(1 << 20)
    while kind in ("append", "attend"):
        sides = rng.choices(("decode", "prefill", "both"), (4, 2, 4))[0]
        lo = _log(rng, 1, 8192)
        hi = _log(rng, lo, 32768)
        decodes = 0 if sides == "prefill" else _log(rng, 1, 256)
        chunks = 0 if sides == "decode" else rng.choice((1, 1, 2, 3, 4, 6))
        most = _log(rng, 2, 2600)
        prior = rng.choice((0, _log(rng, 1, 32768)))
        c = _step("", kind, model, decodes, (lo, hi) if decodes else (0, 0), chunks, (max(2, most // rng.choice((1, 1, 3))), most) if chunks else (0, 0),
                  (0, prior) if chunks else (0, 0), "bf16" if rng.random() < 0.6 else "f16", lengths)
        del c["name"]
        hq, hkv, d, _ = MODELS[model]
        seqs = _lengths(c)
        kv = max(sum(q == 1 for _, q in seqs) * max([x for x, q in seqs if q == 1], default=0),
                 sum(q > 1 for _, q in seqs) * max([x + q for x, q in seqs if q > 1], default=0)) * hkv * d
        scores = sum(q > 1 for _, q in seqs) * max([q * (x + q) for x, q in seqs if q > 1], default=0) * hq
        if work(c)["flops"] <= 1.1e12 and work(c)["bytes"] <= 3.0e9 and kv <= 4.0e9 and scores <= 2.1e9:
            return c
    layers, bits = rng.randint(1, MODELS[model][3]), rng.choice((8, 8, 16))
    while True:
        if kind == "copy":
            c = _pages("", kind, model, layers, bits, lengths, count=_log(rng, 1, 1152))
        elif kind == "fork":
            lo = _log(rng, 1, 1500)
            c = _pages("", kind, model, layers, bits, lengths, parents=_log(rng, 1, 64), children=rng.randint(1, 8), len_lo=lo, len_hi=_log(rng, lo, 2000))
        else:
            lo = _log(rng, 1, 2000)
            rows = _log(rng, 1, 96)
            c = _pages("", kind, model, layers, bits, lengths, rows=rows, prefix=rng.choice((0, 1, 5, 16)), len_lo=lo, len_hi=_log(rng, lo, 4000),
                       spare=_log(rng, 1, 6000), moves=0)
            used, spare = _used(c), c["spare"]
            c["moves"] = min(used, spare, _log(rng, 1, 3100))
        del c["name"]
        w = work(c)["bytes"]
        if w <= 2.0e9 and _num_pages(c) * _page_bytes(c) * layers <= 1.5e10:
            return c
        layers = max(1, layers // 2)


# ---------------------------------------------------------------------------------- sizes

def _lengths(case):
    """(cached tokens, new tokens) of every sequence, the decodes first."""
    r = random.Random(case["lengths"])
    seqs = [(r.randint(case["ctx_lo"], case["ctx_hi"]), 1) for _ in range(case["decodes"])]
    return seqs + [(r.randint(case["prior_lo"], case["prior_hi"]), r.randint(case["chunk_lo"], case["chunk_hi"])) for _ in range(case["chunks"])]


def _row_lengths(case):
    r = random.Random(case["lengths"])
    n = case["parents"] if case["kind"] == "fork" else case["rows"]
    return [r.randint(case["len_lo"], case["len_hi"]) for _ in range(n)]


def _blocks(n):
    return -(-n // PAGE)


def _prefix(case, n):
    """Pages that a row of n tokens shares with the others: full ones only."""
    return min(case["prefix"], n // PAGE)


def _used(case):
    lens = _row_lengths(case)
    return max(_prefix(case, n) for n in lens) + sum(_blocks(n) - _prefix(case, n) for n in lens)


def _num_pages(case):
    if case["kind"] == "copy":
        return 2 * case["count"] + case["count"] // 4 + 8
    if case["kind"] == "fork":
        return sum(_blocks(n) for n in _row_lengths(case)) + case["parents"] * case["children"] + 8
    return _used(case) + case["spare"]


def _page_bytes(case):
    """Of one page and layer: 8-bit codes with their scales, or 16-bit values."""
    _, hkv, d, _ = MODELS[case["model"]]
    return 2 * hkv * (PAGE * d + 4) if case.get("bits", 8) == 8 else 2 * hkv * PAGE * d * 2


def _page_stride(case):
    return -(-_page_bytes(case) // 128) * 128


def work(case):
    hq, hkv, d, _ = MODELS[case["model"]]
    if case["kind"] == "append":
        # the new rows read, their codes written, the scales of the pages they lie in written, the tables read
        nbytes = sum(q * 2 * hkv * d * 3 + (_blocks(c + q) - c // PAGE) * (2 * hkv * 4 + 4) for c, q in _lengths(case))
        return {"bytes": nbytes, "flops": 0}
    if case["kind"] == "attend":
        nbytes = flops = 0
        for c, q in _lengths(case):
            # codes and scales of the sequence and its page table read once, Q read and the output written once
            nbytes += (c + q) * 2 * hkv * d + _blocks(c + q) * (2 * hkv * 4 + 4) + 2 * q * hq * d * 2
            flops += 4 * hq * d * (q * c + q * (q + 1) // 2)
        return {"bytes": nbytes, "flops": flops}
    page = _page_bytes(case) * case["layers"]
    if case["kind"] == "copy":
        return {"bytes": 2 * case["count"] * page + 8 * case["count"], "flops": 0}
    if case["kind"] == "fork":
        # the unfinished last pages copied; tables of parents read, of the children read (free) and written, a count for each entry
        # read and written by either call
        lens = _row_lengths(case)
        entries = sum(_blocks(n) for n in lens)
        return {"bytes": case["children"] * (sum(n % PAGE != 0 for n in lens) * 2 * page + entries * (4 + 4 + 16)) + entries * 4, "flops": 0}
    # the moved pages read and written; counts read and written and a new number written for every page; the tables read and written
    return {"bytes": case["moves"] * 2 * page + 12 * _num_pages(case) + 8 * sum(_blocks(n) for n in _row_lengths(case)), "flops": 0}


# --------------------------------------------------------------------------------- inputs

def _fill8(pool, hkv, d, gen):
    """Codes of N(0, 1) values and scales around 2**-6: pool [..., page stride] bytes."""
    codes = 2 * hkv * PAGE * d
    rows = pool.view(-1, pool.shape[-1])
    for part in rows.split(16384):
        x = torch.randn((part.shape[0], codes), generator=gen, device="cuda") * 64
        part[:, :codes] = x.clamp_(-FP8_MAX, FP8_MAX).to(FP8).view(torch.uint8)
        part[:, codes:codes + 8 * hkv] = torch.exp2(torch.randint(-7, -4, (part.shape[0], 2 * hkv), generator=gen, device="cuda").float()).view(torch.uint8)
        part[:, codes + 8 * hkv:] = 0


def _prepare_step(case, seed):
    hq, hkv, d, _ = MODELS[case["model"]]
    cpu = torch.Generator().manual_seed(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = torch.float16 if case["dtype"] == "f16" else torch.bfloat16
    seqs = _lengths(case)
    need = [_blocks(c + q) for c, q in seqs]
    pages, widest = sum(need), max(need)
    perm = torch.randperm(pages, generator=cpu).to(torch.int32)
    tables = torch.full((len(seqs), widest), -1, dtype=torch.int32)
    tables[torch.arange(widest) < torch.tensor(need)[:, None]] = perm
    ctx = torch.tensor([c for c, _ in seqs], dtype=torch.int32)
    cu = torch.zeros(len(seqs) + 1, dtype=torch.int32)
    cu[1:] = torch.cumsum(torch.tensor([q for _, q in seqs]), 0)
    total = int(cu[-1])
    pool = torch.empty((1, pages, _page_stride(case)), dtype=torch.uint8, device="cuda")
    _fill8(pool, hkv, d, gen)
    state = {"kind": case["kind"], "hq": hq, "hkv": hkv, "d": d, "dtype": dtype, "pool": pool, "decodes": case["decodes"], "seqs": len(seqs),
             "tables": tables.cuda(), "ctx": ctx.cuda(), "cu": cu.cuda(), "scale": 1 / math.sqrt(d),
             # the longest of the decodes and of the chunks, for the sizes of the plain form
             "longest": [max([c + q for c, q in g], default=0) for g in (seqs[:case["decodes"]], seqs[case["decodes"]:])],
             "most_new": [1, max([q for _, q in seqs[case["decodes"]:]], default=0)]}
    if case["kind"] == "append":
        # N(0, 1) rows, each token with a size of its own, a few of them outliers
        gain = torch.exp2(torch.randn((total, 1, 1), generator=gen, device="cuda"))
        state["k"], state["v"] = ((torch.randn((total, hkv, d), generator=gen, device="cuda") * gain).to(dtype) for _ in range(2))
    else:
        state["q"] = torch.randn((total, hq, d), generator=gen, device="cuda", dtype=dtype)
        state["out"] = torch.empty_like(state["q"])
    if own:
        from paper_2410_01228_amd import binding as cs
        state["batch"] = cs.Batch(tables, ctx, cu)
        state["handle"] = cs.Pool8(pool, 1, pages, hkv, d, page_stride=pool.shape[-1])
        if case["kind"] == "attend":
            state["workspace"] = cs.workspace_for_kv8(state["batch"], hq, hkv, d)
    return state


def _prepare_pages(case, seed):
    _, hkv, d, _ = MODELS[case["model"]]
    layers, pages, stride = case["layers"], _num_pages(case), _page_stride(case)
    cpu = torch.Generator().manual_seed(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    pool = torch.empty((layers, pages, stride), dtype=torch.uint8, device="cuda")
    if case["bits"] == 8:
        _fill8(pool, hkv, d, gen)
    else:
        pool.view(torch.bfloat16).normal_(generator=gen)
    state = {"kind": case["kind"], "layers": layers, "pages": pages, "pool": pool}
    perm = torch.randperm(pages, generator=cpu).to(torch.int32)
    if case["kind"] == "copy":
        n = case["count"]
        state.update(src=perm[:n].cuda(), dst=perm[n:2 * n].cuda())
    elif case["kind"] == "fork":
        lens = _row_lengths(case)
        n, each = len(lens), case["children"]
        need = torch.tensor([_blocks(x) for x in lens])
        widest = int(need.max()) + 1
        tables = torch.full((n * (1 + each), widest), -1, dtype=torch.int32)
        tables[:n][torch.arange(widest) < need[:, None]] = perm[:int(need.sum())]
        fresh = perm[int(need.sum()):int(need.sum()) + n * each]
        parents = torch.arange(n, dtype=torch.int32).repeat_interleave(each)
        children = (n + torch.randperm(n * each, generator=cpu)).to(torch.int32)
        lens = torch.tensor(lens, dtype=torch.int32)
        # as the step before left it: the children are there, forked from the same parents
        all_lens = torch.cat([lens, torch.zeros(n * each, dtype=torch.int32)])
        all_lens[children.long()] = lens[parents.long()]
        tables[children.long()] = tables[parents.long()]
        tail = lens[parents.long()] % PAGE != 0
        tables[children.long()[tail], (lens[parents.long()] // PAGE).long()[tail]] = fresh[tail]
        counts = torch.zeros(pages, dtype=torch.int32)
        counts.index_add_(0, tables[tables >= 0].long(), torch.ones(int((tables >= 0).sum()), dtype=torch.int32))
        state.update(tables=tables.cuda(), lens=all_lens.cuda(), counts=counts.cuda(), parents=parents.cuda(), children=children.cuda(), fresh=fresh.cuda(),
                     freed=torch.full((pages,), -1, dtype=torch.int32, device="cuda"), num_freed=torch.zeros(1, dtype=torch.int32, device="cuda"))
    else:
        used, moves = _used(case), case["moves"]
        ids = torch.cat([torch.randperm(used, generator=cpu)[moves:], used + torch.randperm(pages - used, generator=cpu)[:moves]])
        ids = ids[torch.randperm(used, generator=cpu)].to(torch.int32)
        lens = torch.tensor(_row_lengths(case), dtype=torch.int32)
        need, shared = (lens + PAGE - 1) // PAGE, torch.minimum(lens // PAGE, torch.tensor(case["prefix"]))
        widest, first = int(need.max()), int(shared.max())
        at = torch.arange(widest)
        tables = torch.full((len(lens), widest), -1, dtype=torch.int32)
        mine = (at >= shared[:, None]) & (at < need[:, None])
        tables[mine] = ids[first:]
        tables = torch.where(at < shared[:, None], torch.nn.functional.pad(ids[:first], (0, widest - first)), tables)
        counts = torch.zeros(pages, dtype=torch.int32)
        counts.index_add_(0, tables[tables >= 0].long(), torch.ones(int((tables >= 0).sum()), dtype=torch.int32))
        state.update(tables=tables.cuda(), lens=lens.cuda(), counts=counts.cuda(), new_tables=torch.full_like(tables, -1).cuda(), new_counts=torch.zeros_like(counts).cuda(),
                     new_ids=torch.zeros_like(counts).cuda(), num_used=torch.zeros(1, dtype=torch.int32, device="cuda"))
    if own:
        from paper_2410_01228_amd import binding as cs
        if case["bits"] == 8:
            state["space"] = cs.PageSpace.of(cs.Pool8(pool, layers, pages, hkv, d, page_stride=stride))
        else:
            state["space"] = cs.PageSpace.of(cs.Pool(pool, layers, pages, hkv, d, page_stride=stride // 2))
        if case["kind"] != "copy":
            state["rows"] = cs.PageTables(state["tables"], state["lens"], state["counts"])
        if case["kind"] == "compact":
            state["new_rows"] = cs.PageTables(state["new_tables"], state["lens"], state["new_counts"])
            state["workspace"] = cs.compact_workspace_for(state["space"])
    return state


def prepare(case, seed):
    return _prepare_step(case, seed) if case["kind"] in ("append", "attend") else _prepare_pages(case, seed)


# ------------------------------------------------------------------------------ plain forms

def _pool_outputs(s):
    """The pool as the values its codes stand for (times their block's scale), and the scales."""
    codes = 2 * s["hkv"] * PAGE * s["d"]
    return {"codes": s["pool"][..., :codes].view(FP8), "scales": s["pool"][..., codes:codes + 8 * s["hkv"]].view(torch.float32)}


def _blocks_of(s, pages):
    """float32 [..., K/V, kv head, token, feature] codes and [..., K/V, kv head] scales of the pages with these ids."""
    hkv, d = s["hkv"], s["d"]
    raw = s["pool"][0].view(torch.int64)[pages].view(torch.uint8)
    codes, lead = 2 * hkv * PAGE * d, pages.shape
    x = raw[..., :codes].view(FP8).view(*lead, 2, hkv, PAGE * d)
    n = len(lead)
    k = x.select(n, 0).reshape(*lead, hkv, d // 16, PAGE, 16).transpose(-3, -2).reshape(*lead, hkv, PAGE, d)
    v = x.select(n, 1).reshape(*lead, hkv, d // 64, 4, 16, 4, 4).permute(*range(n + 1), n + 2, n + 5, n + 1, n + 4, n + 3).reshape(*lead, hkv, PAGE, d)
    return torch.stack([k, v], n).float(), raw[..., codes:codes + 8 * hkv].view(torch.float32).view(*lead, 2, hkv)


def _exponent_for(top):
    """The least e >= LOWEST_EXPONENT with top <= 448 * 2**e, as integers."""
    m, e = torch.frexp(top)                              # top = m * 2**e, 0.5 <= m < 1; 448 = 0.875 * 2**9
    return torch.where(top > 0, e - 9 + (m > 0.875).to(e.dtype), LOWEST_EXPONENT).clamp_min(LOWEST_EXPONENT)


def _plain_append(s):
    hkv, d, tables, ctx, cu = s["hkv"], s["d"], s["tables"].long(), s["ctx"].long(), s["cu"].long()
    total = s["k"].shape[0]
    token = torch.arange(total, device="cuda")
    seq = torch.searchsorted(cu[1:], token, right=True)
    pos = ctx[seq] + token - cu[seq]
    page, slot = tables[seq, pos // PAGE], pos % PAGE
    new = torch.stack([s["k"], s["v"]], 1).float()                                  # [T, K/V, Hkv, D]
    if s["dtype"] == torch.float16:
        new = new.clamp(-F16_MOST, F16_MOST)
    # the pages of the step, each once: `at` is a token's place among them
    touched = torch.zeros(s["pool"].shape[1], dtype=torch.long, device="cuda").index_fill_(0, page, 1)
    ids = touched.nonzero()[:, 0]
    at = (touched.cumsum(0) - 1)[page]
    fresh = torch.zeros((len(ids), PAGE), dtype=torch.bool, device="cuda")
    fresh[at, slot] = True
    kept = torch.arange(PAGE, device="cuda") < torch.zeros(len(ids), dtype=torch.long, device="cuda").index_add_(
        0, at[(token == cu[seq])], (ctx[seq] % PAGE)[token == cu[seq]])[:, None]     # tokens that the page held before
    old, scale = _blocks_of(s, ids)
    top = torch.zeros((len(ids), 2, hkv), device="cuda").index_reduce_(0, at, new.abs().amax(-1), "amax")
    before = torch.where(kept.any(1)[:, None, None], torch.frexp(scale)[1] - 1, LOWEST_EXPONENT)
    e = torch.maximum(_exponent_for(top), before)
    raised = torch.ldexp(old, (before - e)[..., None, None])                        # the tokens before, at the new scale
    block = torch.where(kept[:, None, None, :, None], raised, old)
    block[at, :, :, slot] = torch.ldexp(new, -e[at][..., None])
    block = block.to(FP8)
    k = block[:, 0].view(-1, hkv, PAGE, d // 16, 16).transpose(2, 3)
    v = block[:, 1].view(-1, hkv, 4, 4, d // 64, 4, 16).permute(0, 1, 4, 2, 6, 5, 3)
    codes = torch.cat([k.reshape(len(ids), -1), v.reshape(len(ids), -1)], 1).view(torch.uint8)
    scales = torch.ldexp(torch.ones_like(scale), e).view(len(ids), -1).view(torch.uint8)
    s["pool"][0, ids, :codes.shape[1] + scales.shape[1]] = torch.cat([codes, scales], 1)
    return _pool_outputs(s)


def _plain_group(s, first, end, longest, most):
    """Sequences first .. end - 1, padded to the longest of them."""
    hq, hkv, d, n = s["hq"], s["hkv"], s["d"], end - first
    ctx, cu, out = s["ctx"].long()[first:end], s["cu"].long()[first:end + 1], s["out"]
    blocks, scales = _blocks_of(s, s["tables"][first:end, :_blocks(longest)].long().clamp_min(0))
    blocks *= scales[..., None, None]
    k, v = (blocks[:, :, i].transpose(1, 2).reshape(n, hkv, -1, d) for i in (0, 1))
    del blocks
    new = torch.arange(most, device="cuda")
    token = (cu[:-1, None] + new).clamp_max(s["q"].shape[0] - 1)
    q = s["q"][token].float().view(n, most, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, -1, d)
    key = torch.arange(k.shape[2], device="cuda")
    v = torch.where((key < (ctx + cu[1:] - cu[:-1])[:, None])[:, None, :, None], v, torch.zeros((), device="cuda"))
    x = torch.matmul(q, k.transpose(2, 3)).view(n, hkv, hq // hkv, most, -1).mul_(s["scale"])
    x.masked_fill_((key > (ctx[:, None] + new)[..., None])[:, None, None], -math.inf)
    x -= x.amax(-1, keepdim=True)
    x.exp_()
    y = torch.matmul(x.view(n, hkv, -1, x.shape[-1]), v).view(n, hkv, hq // hkv, most, d) / x.sum(-1, keepdim=True)
    there = new < (cu[1:] - cu[:-1])[:, None]
    out[token[there]] = y.permute(0, 3, 1, 2, 4).reshape(n, most, hq, d)[there].to(out.dtype)


def _plain_attend(s):
    if s["decodes"]:
        _plain_group(s, 0, s["decodes"], s["longest"][0], 1)
    if s["seqs"] > s["decodes"]:
        _plain_group(s, s["decodes"], s["seqs"], s["longest"][1], s["most_new"][1])
    return s["out"]


def _entries(s, rows):
    """Ids in these rows of the tables, one past the last page where a row has none."""
    t = s["tables"][rows]
    there = torch.arange(t.shape[1], device="cuda") < ((s["lens"][rows] + PAGE - 1) // PAGE)[:, None]
    return torch.where(there, t, s["pages"]).long()


def _plain_fork(s):
    pages, counts, pool = s["pages"], s["counts"], s["pool"].view(torch.int64)
    children, parents = s["children"].long(), s["parents"].long()
    one = torch.ones((), dtype=torch.int32, device="cuda")
    # the losers leave: a page that nobody else holds is free again, and listed
    gone = _entries(s, children).view(-1)
    left = counts - torch.zeros(pages + 1, dtype=torch.int32, device="cuda").index_add_(0, gone, one.expand(len(gone)))[:pages]
    free = (counts > 0) & (left == 0)
    place = torch.where(free, free.cumsum(0) - 1, pages)
    listed_ = torch.cat([s["freed"], s["freed"][:1]])
    listed_[place] = torch.arange(pages, dtype=torch.int32, device="cuda")
    s["freed"].copy_(listed_[:pages])
    s["num_freed"].copy_(free.sum())
    counts.copy_(left)
    s["tables"][children] = -1
    s["lens"][children] = 0
    # the winners' children: full pages shared, the last one copied if it has room
    lens = s["lens"][parents]
    row = s["tables"][parents]
    last = (lens // PAGE).long()
    tail = lens % PAGE != 0
    src, dst = row[tail, last[tail]].long(), s["fresh"][tail]
    row[tail, last[tail]] = dst
    at = torch.arange(row.shape[1], device="cuda")
    s["tables"][children] = torch.where(at < ((lens + PAGE - 1) // PAGE)[:, None], row, -1)
    s["lens"][children] = lens
    held = _entries(s, children).view(-1)
    counts += torch.zeros(pages + 1, dtype=torch.int32, device="cuda").index_add_(0, held, one.expand(len(held)))[:pages]
    pool[:, dst.long()] = pool[:, src]
    return _fork_outputs(s)


def _fork_outputs(s):
    return {"tables": s["tables"], "lens": s["lens"], "counts": s["counts"], "freed": s["freed"], "num_freed": s["num_freed"], "pool": s["pool"].view(torch.int32)}


def _plain_compact(s):
    pages, counts, pool = s["pages"], s["counts"], s["pool"].view(torch.int64)
    at = torch.arange(pages, dtype=torch.int32, device="cuda")
    used = counts > 0
    n = used.sum()
    src, dst = (used & (at >= n)).nonzero()[:, 0], (~used & (at < n)).nonzero()[:, 0]
    ids = torch.where(used, at, -1)
    ids[src] = dst.to(torch.int32)
    s["new_ids"].copy_(ids)
    s["new_counts"].zero_()
    s["new_counts"][ids[used].long()] = counts[used]
    there = torch.arange(s["tables"].shape[1], device="cuda") < ((s["lens"] + PAGE - 1) // PAGE)[:, None]
    s["new_tables"].copy_(torch.where(there, ids[s["tables"].clamp_min(0).long()], -1))
    s["num_used"].copy_(n)
    pool[:, dst] = pool[:, src]
    return _compact_outputs(s)


def _compact_outputs(s):
    return {"tables": s["new_tables"], "counts": s["new_counts"], "new_ids": s["new_ids"], "num_used": s["num_used"], "pool": s["pool"].view(torch.int32)}


def run(state):
    s, kind = state, state["kind"]
    if not own:
        if kind == "append":
            return _plain_append(s)
        if kind == "attend":
            return _plain_attend(s)
        if kind == "fork":
            return _plain_fork(s)
        if kind == "compact":
            return _plain_compact(s)
        pool = s["pool"].view(torch.int64)
        pool[:, s["dst"].long()] = pool[:, s["src"].long()]
        return s["pool"].view(torch.int32)
    from paper_2410_01228_amd import binding as cs
    if kind == "append":
        append = cs.cs_kv8_append_f16 if s["dtype"] == torch.float16 else cs.cs_kv8_append
        append(s["handle"], 0, s["batch"], s["k"], s["v"])
        return _pool_outputs(s)
    if kind == "attend":
        attend = cs.cs_paged_attention_mixed_kv8_f16 if s["dtype"] == torch.float16 else cs.cs_paged_attention_mixed_kv8
        attend(s["handle"], 0, s["batch"], s["q"], s["out"], s["hq"], s["scale"], s["workspace"])
        return s["out"]
    if kind == "copy":
        cs.cs_kv_pages_copy(s["space"], 0, s["src"], s["space"], 0, s["dst"], s["layers"])
        return s["pool"].view(torch.int32)
    if kind == "fork":
        cs.cs_kv_pages_free(s["rows"], s["children"], s["freed"], s["num_freed"])
        cs.cs_kv_pages_fork(s["space"], 0, s["layers"], s["rows"], s["parents"], s["children"], s["fresh"])
        return _fork_outputs(s)
    cs.cs_kv_pages_compact(s["space"], 0, s["layers"], s["rows"], s["new_rows"], s["new_ids"], s["num_used"], s["workspace"])
    return _compact_outputs(s)


# -------------------------------------------------------------------------- 64-bit definition

def _code_values():
    """What the 256 codes of e4m3 stand for: 1 sign, 4 exponent (bias 7), 3 mantissa bits; 127 and 255 are not numbers."""
    v = []
    for c in range(128):
        e, m = c >> 3, c & 7
        v.append(math.nan if c == 127 else math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10))
    return torch.tensor(v + [-x for x in v], dtype=torch.float64, device="cuda")


def _nearest_code(x):
    """x (float64, at most 448 in size) rounded to the nearest e4m3 value, ties to the even one: steps of 2**(e - 3) from 2**e on, 2**-9 below 2**-6."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _where(d):
    """Code numbers of K and V inside their blocks, [token, feature] each."""
    t, f = torch.arange(PAGE, device="cuda")[:, None], torch.arange(d, device="cuda")
    return (f // 16 * 16 + t) * 16 + f % 16, ((f // 64 * 4 + t // 4) * 16 + f % 16) * 16 + f // 16 % 4 * 4 + t % 4


def _exact_append(case, s):
    hkv, d = s["hkv"], s["d"]
    where, value, codes = _where(d), _code_values(), 2 * hkv * PAGE * d
    pool = s["pool"][0]
    block = value[pool[:, :codes].long()].view(-1, 2, hkv, PAGE * d)
    scale = pool[:, codes:codes + 8 * hkv].reshape(-1, 2 * hkv * 4).view(torch.float32).double().view(-1, 2, hkv)
    most = F16_MOST if case["dtype"] == "f16" else math.inf
    t0 = 0
    for i, (c, q) in enumerate(_lengths(case)):
        for j in range(c // PAGE, _blocks(c + q)):
            lo, hi = max(c, j * PAGE), min(c + q, j * PAGE + PAGE)
            p, held = int(s["tables"][i, j]), max(0, lo - j * PAGE)
            for kv, rows in enumerate((s["k"], s["v"])):
                x = rows[t0 + lo - c:t0 + hi - c].double().clamp(-most, most)          # [tokens, Hkv, D]
                e = torch.ceil(torch.log2(x.abs().amax((0, 2)).clamp_min(1e-300) / FP8_MAX)).clamp_min(LOWEST_EXPONENT)
                if held:
                    e = torch.maximum(e, torch.log2(scale[p, kv]))
                at = where[kv]
                if held:
                    old = block[p, kv][:, at[:held]] * (scale[p, kv] / torch.exp2(e))[:, None, None]
                    block[p, kv][:, at[:held]] = _nearest_code(old)
                block[p, kv][:, at[lo - j * PAGE:hi - j * PAGE]] = _nearest_code(x.transpose(0, 1) / torch.exp2(e)[:, None, None])
                scale[p, kv] = torch.exp2(e)
        t0 += q
    return {"codes": block.view(1, -1, codes), "scales": scale.view(1, -1, 2 * hkv)}


def _exact_attend(case, s):
    hq, hkv, d = s["hq"], s["hkv"], s["d"]
    where, value, codes = _where(d), _code_values(), 2 * hkv * PAGE * d
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    t0 = 0
    for i, (c, q) in enumerate(_lengths(case)):
        raw = s["pool"][0, s["tables"][i, :_blocks(c + q)].long()]
        scale = raw[:, codes:codes + 8 * hkv].contiguous().view(torch.float32).double().view(-1, 2, hkv)
        raw = raw[:, :codes].reshape(-1, 2, hkv, PAGE * d)
        for g in range(hkv):
            k, v = ((value[raw[:, kv, g].long()][:, where[kv]] * scale[:, kv, g, None, None]).reshape(-1, d)[:c + q] for kv in (0, 1))
            for r in range(0, q, 512):
                rows = s["q"][t0 + r:t0 + min(q, r + 512), g * (hq // hkv):(g + 1) * (hq // hkv)].double()
                x = torch.matmul(rows.transpose(0, 1), k.T) / math.sqrt(d)
                late = torch.arange(c + q, device="cuda") > (c + r + torch.arange(rows.shape[0], device="cuda"))[:, None]
                x = torch.softmax(x.masked_fill(late, -math.inf), -1)
                out[t0 + r:t0 + r + rows.shape[0], g * (hq // hkv):(g + 1) * (hq // hkv)] = torch.matmul(x, v).transpose(0, 1)
        t0 += q
    return out


def exact(case, seed):
    if case["kind"] not in ("append", "attend"):
        return None                                      # bytes and page numbers: nothing is computed
    s = _prepare_step(case, seed)
    return _exact_append(case, s) if case["kind"] == "append" else _exact_attend(case, s)
