"""The paged compressed KV cache: slots and block tables from request lengths, new tokens into pages, attention out of them.

A case is a dict of plain values; `op` says which operator one pass goes through:

  plan     ecco_paged_plan: every request's new tokens get slots, pages that are missing come from a list of free ones
  append   ecco_paged_append: K and V rows of new tokens, compressed to 64-byte blocks, into the slots of their tokens
  attn     ecco_paged_attn: each request's new tokens attend to the request's pages (causal: the new tokens are the cache's
           last; otherwise, as with an encoder's states, every new token sees all of it)

The plain forms below decode and encode the block format (64 bytes for 128 fp16 values: E4M3 scale, codebook id, Huffman-coded
pattern id, 128 Huffman-coded indices, outliers in what is left) with elementary operations on whole tensors.  Values beyond
fp16's range enter the attention as +-65504.  K are N(0,1) with four channels of every head ten times as large, V are N(0,1);
both are scaled as the codec's min/max calibration of such caches has them.  Large pools are filled with blocks
drawn from a bank that was encoded for them, so that they are quick to make.
"""
from __future__ import annotations

import functools
import heapq
import math
import random

import numpy as np
import torch

own = False                 # true: the framework's operators instead of the plain forms

GROUP, BLOCK_BYTES, BLOCK_BITS = 128, 64, 512
PATTERNS, CODEBOOKS, EXPONENT = 64, 4, -3
BANK = 65536                # distinct groups of a large pool
TILE = 32                   # tokens to a tile of a plan's kv_tiles
HALF_MAX = 65504.0


def listed():
    return [
        # A decode step of 64 running requests: one token each, now and then a page.
        {"name": "plan_decode", "op": "plan", "requests": 64, "new": "1-1", "ctx": "0-4095", "page": 16, "len_seed": 1},
        # 2048 requests of a loaded server, some decoding, some with a piece of a prompt, 130 thousand slots.
        {"name": "plan_many", "op": "plan", "requests": 2048, "new": "0-128", "ctx": "0-8191", "page": 32, "len_seed": 2},
        # K and V rows of one new token for 32 sequences with eight KV heads: once per layer and decode step.
        {"name": "append_step", "op": "append", "tokens": 32, "skipped": 0, "kv_heads": 8, "page": 16},
        # A batch padded to a fixed size for a captured graph: 777 tokens, 90 of them padding.
        {"name": "append_padded", "op": "append", "tokens": 777, "skipped": 90, "kv_heads": 8, "page": 64},
        # The prompts of eight sequences of 512 tokens, 32 heads.
        {"name": "append_prefill", "op": "append", "tokens": 4096, "skipped": 0, "kv_heads": 32, "page": 64},
        # Early in two conversations: the smallest decode step.
        {"name": "attn_step_short", "op": "attn", "requests": 2, "new": "1-1", "ctx": "770-783", "kv_heads": 8, "q_per_kv": 4,
         "page": 16, "causal": True, "len_seed": 3},
        # Decode step without grouped heads, eight sequences near 4096 tokens.
        {"name": "attn_step_mha", "op": "attn", "requests": 8, "new": "1-1", "ctx": "4000-4095", "kv_heads": 32, "q_per_kv": 1,
         "page": 64, "causal": True, "len_seed": 4},
        # Decode step of 32 requests of all lengths up to 16384: the largest cache.
        {"name": "attn_step_ragged", "op": "attn", "requests": 32, "new": "1-1", "ctx": "1-16383", "kv_heads": 8, "q_per_kv": 8,
         "page": 32, "causal": True, "len_seed": 5},
        # Four to eight drafted tokens of each of sixteen requests on their way through the target.
        {"name": "attn_drafts", "op": "attn", "requests": 16, "new": "4-8", "ctx": "10-4095", "kv_heads": 8, "q_per_kv": 4,
         "page": 16, "causal": True, "len_seed": 6},
        # A server's mixed batch: mostly single tokens, some pieces of prompts.
        {"name": "attn_mixed", "op": "attn", "requests": 24, "new": "1-1+1-1+1-1+1-500", "ctx": "0-3000", "kv_heads": 8, "q_per_kv": 4,
         "page": 16, "causal": True, "len_seed": 7},
        # The last 2048 tokens of each of two prompts of about 8000: the most arithmetic.
        {"name": "attn_chunk_long", "op": "attn", "requests": 2, "new": "2048-2048", "ctx": "5900-6144", "kv_heads": 8, "q_per_kv": 4,
         "page": 64, "causal": True, "len_seed": 8},
        # A decoder's prompt over an encoder's 1500 states.
        {"name": "attn_cross", "op": "attn", "requests": 8, "new": "3-64", "ctx": "700-1500", "kv_heads": 12, "q_per_kv": 1,
         "page": 64, "causal": False, "len_seed": 9},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "append", "attn", "attn", "attn", "attn"])
    page = rng.choice([1, 8, 16, 16, 32, 64, 128])
    if op == "plan":
        ctx = _log_int(rng, 1, 8192)
        return {"op": op, "requests": _log_int(rng, 1, 2048), "new": "%d-%d" % (rng.randint(0, 1), _log_int(rng, 1, 128)),
                "ctx": "%d-%d" % (rng.randint(0, ctx), ctx), "page": page, "len_seed": rng.randrange(1 << 30)}
    if op == "append":
        heads = rng.choice([1, 2, 4, 8, 8, 16, 32])
        tokens = _log_int(rng, 1, 131072 // heads)
        return {"op": op, "tokens": tokens, "skipped": rng.randint(0, tokens // 4), "kv_heads": heads, "page": page}
    heads = rng.choice([1, 2, 4, 8, 8, 12, 32])
    q_per_kv = rng.choice([1, 1, 2, 3, 4, 4, 5, 8, 8])
    causal = rng.random() < 0.8
    if rng.random() < 0.6:                                             # decode steps and drafts
        new = rng.choice([1, 1, 1, 2, 5, 9])
        ctx = _log_int(rng, 1, 16384)
        requests = max(1, min(_log_int(rng, 1, 64), 2_000_000 // (heads * (ctx + new))))
        new = "%d-%d" % (1 if rng.random() < 0.5 else new, new)
    else:                                                              # pieces of prompts
        new = _log_int(rng, 10, 2048)
        ctx = _log_int(rng, 1, 6144)
        requests = max(1, min(_log_int(rng, 1, 16), 500_000_000 // (heads * q_per_kv * new * (ctx + new)), 130_000 // (heads * (ctx + new))))
        new = "%d-%d" % (rng.randint(1, new), new)
    return {"op": op, "requests": requests, "new": new, "ctx": "%d-%d" % (rng.randint(1, ctx), ctx), "kv_heads": heads, "q_per_kv": q_per_kv,
            "page": page, "causal": causal, "len_seed": rng.randrange(1 << 30)}


# ------------------------------------------------------------------ lengths: they belong to the case, not to the seed
def _lengths(case):
    rng = random.Random(case["len_seed"])
    news = [tuple(map(int, part.split("-"))) for part in case["new"].split("+")]
    lo, hi = map(int, case["ctx"].split("-"))
    new = [rng.randint(*news[i % len(news)]) for i in range(case["requests"])]
    return np.array(new, dtype=np.int64), np.array([rng.randint(lo, hi) for _ in new], dtype=np.int64)


def _seen(new, ctx, causal):
    """Tokens of the cache, and pairs of a query and a token that it sees, over all requests."""
    kv = ctx + new if causal else ctx
    pairs = (new * ctx + new * (new + 1) // 2) if causal else new * ctx
    return kv, int(pairs.sum())


def work(case):
    if case["op"] == "append":
        written = (case["tokens"] - case["skipped"]) * case["kv_heads"]
        return {"bytes": 2 * written * (2 * GROUP + BLOCK_BYTES) + 4 * case["tokens"], "flops": 0}
    new, ctx = _lengths(case)
    if case["op"] == "plan":
        pages = -(-(ctx + new) // case["page"]) - -(-ctx // case["page"])
        touched = (ctx % case["page"] > 0) & (new > 0)                 # table entries read: of pages that are partly filled
        return {"bytes": int(4 * (2 * len(new) + 2 * pages.sum() + touched.sum() + new.sum() + 3 * len(new))), "flops": 0}
    kv, pairs = _seen(new, ctx, case["causal"])
    heads, q_heads = case["kv_heads"], case["kv_heads"] * case["q_per_kv"]
    pages = -(-kv // case["page"])
    return {"bytes": int(2 * BLOCK_BYTES * kv.sum() * heads + new.sum() * q_heads * (2 * GROUP * 2 + 4) + 4 * pages.sum() + 8 * len(new)),
            "flops": 4 * GROUP * q_heads * pairs}


# ------------------------------------------------------------------ metadata: patterns and codebooks of a cache
def _code_lengths(p):
    """Huffman code lengths of sixteen symbols, all of 2 to 8 bits."""
    p = np.asarray(p, dtype=np.float64)
    p = p / p.sum()
    while True:
        heap = [(float(x), i, (i,)) for i, x in enumerate(p)]
        heapq.heapify(heap)
        length = np.zeros(len(p), dtype=np.int64)
        tie = len(p)
        while len(heap) > 1:
            a, b = heapq.heappop(heap), heapq.heappop(heap)
            for s in a[2] + b[2]:
                length[s] += 1
            heapq.heappush(heap, (a[0] + b[0], tie, a[2] + b[2]))
            tie += 1
        if length.min() >= 2 and length.max() <= 8:
            return length
        p = (p + 1.0 / len(p)) / 2


def _codewords(length):
    """Canonical codewords (by length, then symbol), first bit in bit 0."""
    out, code, last = np.zeros(len(length), dtype=np.int64), 0, 0
    for s in sorted(range(len(length)), key=lambda s: (length[s], s)):
        code <<= int(length[s]) - last
        last = int(length[s])
        out[s] = int(format(code, "0%db" % last)[::-1], 2)
        code += 1
    return out


def _rows(kind, shape, gen):
    x = torch.randn(shape, generator=gen, device=gen.device)
    if kind == "k":
        x[..., 3::32] *= 10
    return x.half()


@functools.lru_cache(maxsize=None)
def _tables(kind):
    """Patterns and code lengths of a kind of cache, the same in every run: what a calibration leaves behind."""
    gen = torch.Generator()
    gen.manual_seed(17 if kind == "k" else 18)
    x = _rows(kind, (4096, GROUP), gen).double().numpy()
    top = np.abs(x).argmax(1)
    # the 127 values beside the largest, as parts of it, ascending
    u = np.sort(np.where(np.arange(GROUP) == top[:, None], 2.0, x / np.abs(x).max(1, keepdims=True)), axis=1)[:, :GROUP - 1]
    edges = np.linspace(0, GROUP - 1, 16).astype(int)
    means = np.stack([u[:, a:b].mean(1) for a, b in zip(edges[:-1], edges[1:])], axis=1)
    means[:, 0], means[:, -1] = (means[:, 0] + u[:, 0]) / 2, (means[:, -1] + u[:, -1]) / 2
    order = np.argsort(u[:, -1] - u[:, 0], kind="stable")
    patterns = np.sort(means[order[np.linspace(0, 4095, PATTERNS).astype(int)]], axis=1).astype(np.float16)
    ends = patterns[:, [0, 14]].astype(np.float64)
    chosen = ((ends[None] - u[:, None, [0, -1]]) ** 2).sum(2).argmin(1)
    sym = np.abs(u[:, :, None] - patterns[chosen].astype(np.float64)[:, None]).argmin(2)
    count = np.apply_along_axis(np.bincount, 1, sym, minlength=16) + (np.arange(16) == 15)
    length = np.zeros((PATTERNS, CODEBOOKS, 16), dtype=np.int64)
    use = np.zeros(PATTERNS)
    for k in range(PATTERNS):
        mine = count[chosen == k]
        mine = mine[np.argsort(mine[:, :7].sum(1) - mine[:, 8:15].sum(1), kind="stable")]
        use[k] = len(mine)
        for h in range(CODEBOOKS):
            part = mine[len(mine) * h // CODEBOOKS:len(mine) * (h + 1) // CODEBOOKS]
            length[k, h] = _code_lengths(part.sum(0) + 0.5 + (8.0 if not len(part) else 0.0))
    kp_length = np.empty(PATTERNS, dtype=np.int64)
    kp_length[np.argsort(-use, kind="stable")] = [5] * 16 + [6] * 16 + [7] * 32          # Kraft sum 1
    code = np.stack([_codewords(length[k, h]) for k in range(PATTERNS) for h in range(CODEBOOKS)])
    return {"patterns": patterns, "length": length, "kp_length": kp_length, "code": code, "kp_code": _codewords(kp_length)}


@functools.lru_cache(maxsize=None)
def _device_tables(kind):
    t = _tables(kind)
    length, code = t["length"].reshape(-1, 16), t["code"]
    window = np.zeros((PATTERNS * CODEBOOKS, 256), dtype=np.int64)
    for s in range(16):
        hit = (np.arange(256)[None] & ((1 << length[:, s, None]) - 1)) == code[:, s, None]
        window[hit] = np.broadcast_to((length[:, s] << 4 | s)[:, None], window.shape)[hit]
    kp_window = np.zeros(4096, dtype=np.int64)
    for k in range(PATTERNS):
        kp_window[(np.arange(4096) & ((1 << t["kp_length"][k]) - 1)) == t["kp_code"][k]] = k | int(t["kp_length"][k]) << 8
    byte = np.arange(256)
    exp, man = (byte >> 3) & 15, byte & 7
    fp8 = np.where(exp == 0, man * 2.0 ** -9, (1 + man / 8.0) * 2.0 ** (exp - 7.0)) * np.where(byte & 128, -1.0, 1.0)
    to = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    return {"window": to(window).view(-1), "kp_window": to(kp_window), "fp8": to(fp8.astype(np.float32)),
            "centroids": to(np.concatenate([t["patterns"], np.ones((PATTERNS, 1), np.float16)], 1)).float(),
            "length": to(length).view(-1), "code": to(code).view(-1), "kp_length": to(t["kp_length"]), "kp_code": to(t["kp_code"])}


# ------------------------------------------------------------------ plain forms of the block format
def _half(x):
    return x.clamp(-HALF_MAX, HALF_MAX).half().float()


def _decode(blocks, tab):
    """uint8 [n][64] -> fp32 [n][128], the values that the blocks stand for."""
    if len(blocks) > 524288:
        return torch.cat([_decode(part, tab) for part in blocks.split(524288)])
    n, dev = len(blocks), blocks.device
    words = torch.zeros((n, 18), dtype=torch.int64, device=dev)
    words[:, :16] = blocks.contiguous().view(torch.int32).long() & 0xffffffff
    head = words[:, 0]
    kp = tab["kp_window"][head >> 10 & 0xfff]
    book = ((kp & 0xff) * CODEBOOKS + (head >> 8 & 3)) * 256
    pos = 10 + (kp >> 8)
    scale = tab["fp8"][head & 0xff] * 2.0 ** EXPONENT
    value = torch.zeros((n, 17), device=dev)
    value[:, :16] = _half(tab["centroids"][kp & 0xff] * scale.abs()[:, None])
    value[:, 15] = _half(scale)
    index = torch.empty((n, GROUP), dtype=torch.int64, device=dev)
    there = torch.ones(n, dtype=torch.bool, device=dev)
    for i in range(GROUP):
        at = (pos >> 5)[:, None]
        pair = words.gather(1, at) | words.gather(1, at + 1) << 32
        entry = tab["window"][book + (pair[:, 0] >> (pos & 31) & 0xff)]
        there &= pos + (entry >> 4) <= BLOCK_BITS
        index[:, i] = torch.where(there, entry & 15, 16)
        pos = torch.where(there, pos + (entry >> 4), pos)
    out = value.gather(1, index)
    pads = torch.where(there, (BLOCK_BITS - pos) // 15, 0)
    for j in range(16):
        first = BLOCK_BITS - 15 * (j + 1)
        field = (words[:, first >> 5] | words[:, (first >> 5) + 1] << 32) >> (first & 31) & 0x7fff
        place = (field & 127)[:, None]
        outlier = _half(tab["fp8"][field >> 7] * 2.0 ** EXPONENT)
        out.scatter_(1, place, torch.where(pads > j, outlier, out.gather(1, place)[:, 0])[:, None])
    return out


def _to_fp8(x):
    return (x * 2.0 ** -EXPONENT).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).long()


def _encode(x, tab):
    """fp16 [n][128] -> uint8 [n][64], min/max pattern choice; ties go to the lowest index."""
    if len(x) > 65536:
        return torch.cat([_encode(part, tab) for part in x.split(65536)])
    n, dev = len(x), x.device
    place = torch.arange(GROUP, device=dev)
    key = (x.view(torch.int16).long() & 0x7fff) << 7 | (127 - place)
    top = 127 - (key.amax(1) & 127)
    is_top = place == top[:, None]
    x = x.float()
    scale_byte = _to_fp8(x.gather(1, top[:, None]))[:, 0]
    scale = (tab["fp8"][scale_byte] * 2.0 ** EXPONENT).abs().double()[:, None]
    # the quotient in 64 bits, rounded to 32: a division in 32 bits would have to be correctly rounded
    u = torch.where(is_top | (scale == 0), 0.0, (x.double() / torch.where(scale == 0, 1.0, scale)).float()).double()
    low = torch.where(is_top, math.inf, u).amin(1, keepdim=True)
    high = torch.where(is_top, -math.inf, u).amax(1, keepdim=True)
    centroids = tab["centroids"].double()
    off0, off1 = centroids[:, 0] - low, centroids[:, 14] - high
    kp = (off0 * off0 + off1 * off1).argmin(1)
    best = torch.full_like(u, math.inf)
    sym = torch.zeros_like(key)
    for s in range(15):
        d = u - centroids[kp, s, None]
        d = d * d
        sym = torch.where(d < best, s, sym)
        best = torch.minimum(best, d)
    sym = torch.where(is_top, 15, sym)
    total = torch.stack([tab["length"][(kp * CODEBOOKS + h)[:, None] * 16 + sym].sum(1) for h in range(CODEBOOKS)], 1)
    hf = total.argmin(1)
    entry = (kp * CODEBOOKS + hf)[:, None] * 16 + sym
    length, code = tab["length"][entry], tab["code"][entry]
    first = 10 + tab["kp_length"][kp]
    start = first[:, None] + length.cumsum(1) - length
    words = torch.zeros((n, 17), dtype=torch.int64, device=dev)         # 32 bits to a word; sums of bits that are set once
    words[:, 0] = scale_byte | hf << 8 | tab["kp_code"][kp] << 10

    def put(start, bits, count):
        """Bits of a value from a place on, what lies behind the block's end dropped."""
        bits = bits & ((1 << (BLOCK_BITS - start).clamp(min=0).minimum(count)) - 1)
        at = (start >> 5).clamp(max=15)
        bits = bits << (start & 31)
        words.scatter_add_(1, at, bits & 0xffffffff)
        words.scatter_add_(1, at + 1, bits >> 32)

    put(start, code, length)
    end = first + length.sum(1)
    pads = torch.where(end <= BLOCK_BITS, ((BLOCK_BITS - end) // 15).clamp(max=16), 0)
    order = torch.where(is_top, -1, key).topk(16, dim=1).indices
    slot = torch.arange(16, device=dev)
    field = order | _to_fp8(x).gather(1, order) << 7
    used = slot < pads[:, None]
    put((BLOCK_BITS - 15 * (slot + 1)).expand(n, 16), torch.where(used, field, 0), torch.full_like(field, 15))
    return words[:, :16].contiguous().view(torch.int32)[:, ::2].contiguous().view(torch.uint8)


# ------------------------------------------------------------------ what a program has in hand
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def _pool(kind, pages, heads, page, gen):
    n = pages * heads * page
    bank = _encode(_rows(kind, (min(n, BANK), GROUP), gen), _device_tables(kind))
    pick = torch.randint(len(bank), (n,), generator=gen, device="cuda")
    return bank[pick].view(pages, heads, page, BLOCK_BYTES)


def _image(kind):
    """The metadata image that the framework's calls read."""
    from paper_2505_06901_b200 import binding as B

    t = _tables(kind)
    return B.meta_to_device(B.ecco_meta_create(PATTERNS, EXPONENT, t["patterns"], t["length"].astype(np.uint8), t["kp_length"].astype(np.uint8)))


def _cache(st, case, pages, gen):
    heads, page = case["kv_heads"], case["page"]
    st["k"], st["v"] = _pool("k", pages, heads, page, gen), _pool("v", pages, heads, page, gen)
    if own:
        from paper_2505_06901_b200 import binding as B

        st["k_meta"], st["v_meta"] = _image("k"), _image("v")
        st["cache"] = B.paged_cache(st["k_meta"], st["v_meta"], st["k"], st["v"], pages, heads, page)
    else:
        st["k_tab"], st["v_tab"] = _device_tables("k"), _device_tables("v")


def prepare(case, seed):
    gen = _generator(seed)
    st = {"case": case}
    if case["op"] == "plan":
        new, ctx = _lengths(case)
        page, n = case["page"], len(new)
        held, need = -(-ctx // page), -(-(ctx + new) // page) - -(-ctx // page)
        pages = int(held.sum() + need.sum()) + 64
        order = torch.randperm(pages, generator=gen, device="cuda").int()
        st["stride"] = int((held + need).max()) + 3
        tables = torch.full((n, st["stride"]), -1, dtype=torch.int32, device="cuda")
        column = torch.arange(st["stride"], device="cuda")
        tables[column < _ints(held)[:, None]] = order[:int(held.sum())]
        st.update(tables=tables, free=order[int(held.sum()):].contiguous(), pages=pages, new=_ints(new), ctx=_ints(ctx),
                  slots=torch.zeros(int(new.sum()) + 5, dtype=torch.int32, device="cuda"),
                  cu_new=torch.zeros(n + 1, dtype=torch.int32, device="cuda"), kv_lens=torch.zeros(n, dtype=torch.int32, device="cuda"),
                  kv_tiles=torch.zeros(n + 1, dtype=torch.int32, device="cuda"), result=torch.zeros(4, dtype=torch.int32, device="cuda"))
    elif case["op"] == "append":
        tokens, heads, page = case["tokens"], case["kv_heads"], case["page"]
        pages = -(-tokens * 3 // (2 * page)) + 2
        slots = torch.randperm(pages * page, generator=gen, device="cuda")[:tokens].int()
        slots[torch.randperm(tokens, generator=gen, device="cuda")[:case["skipped"]]] = -1
        _cache(st, case, pages, gen)
        # K and V as parts of the rows that one projection writes: queries (as many heads again), keys, values
        qkv = torch.empty((tokens, 3 * heads, GROUP), dtype=torch.float16, device="cuda")
        qkv[:, heads:2 * heads], qkv[:, 2 * heads:] = _rows("k", (tokens, heads, GROUP), gen), _rows("v", (tokens, heads, GROUP), gen)
        qkv[:, :heads] = 0
        st.update(qkv=qkv, slots=slots)
    else:
        new, ctx = _lengths(case)
        kv, _ = _seen(new, ctx, case["causal"])
        page, n = case["page"], len(new)
        held = -(-kv // page)
        pages = int(held.sum()) + 7
        st["stride"] = int(held.max()) + 1
        tables = torch.full((n, st["stride"]), -1, dtype=torch.int32, device="cuda")
        tables[torch.arange(st["stride"], device="cuda") < _ints(held)[:, None]] = torch.randperm(pages, generator=gen, device="cuda").int()[:int(held.sum())]
        _cache(st, case, pages, gen)
        heads, q_per_kv, tokens = case["kv_heads"], case["q_per_kv"], int(new.sum())
        tiles = np.concatenate([[0], np.cumsum(-(-kv // TILE))])
        st.update(tables=tables, kv_lens=_ints(kv), kv_tiles=_ints(tiles), cu_new=_ints(np.concatenate([[0], np.cumsum(new)])),
                  q=torch.randn((tokens, heads * q_per_kv, GROUP), generator=gen, device="cuda").half(),
                  new_host=new.tolist(), kv_host=kv.tolist(), scale=GROUP ** -0.5)
        if own:
            from paper_2505_06901_b200 import binding as B

            st["batch"] = B.paged_batch(tables, st["stride"], st["cu_new"], st["kv_lens"], st["kv_tiles"], n, tokens, int(new.max()), int(kv.max()), int(tiles[-1]))
            st["ws_bytes"] = B.ecco_paged_attn_workspace_bytes(st["cache"], st["batch"], q_per_kv)
            st["ws"] = torch.empty(st["ws_bytes"], dtype=torch.uint8, device="cuda")
            st["out"] = torch.empty((tokens, heads * q_per_kv, GROUP), dtype=torch.float16, device="cuda")
            st["lse"] = torch.empty((tokens, heads * q_per_kv), device="cuda")
    return st


# ------------------------------------------------------------------ one pass
def _plan(st):
    page, n = st["case"]["page"], len(st["new"])
    ctx, new = st["ctx"].long(), st["new"].long()
    held, total = (ctx + page - 1) // page, (ctx + new + page - 1) // page
    need = total - held
    before = need.cumsum(0) - need
    column = torch.arange(st["stride"], device="cuda")
    take = (before[:, None] + column - held[:, None]).clamp(0, len(st["free"]) - 1)
    fresh = (column >= held[:, None]) & (column < total[:, None])
    st["tables"].copy_(torch.where(fresh, st["free"][take], st["tables"]))
    st["cu_new"][1:] = new.cumsum(0)
    st["kv_lens"].copy_(ctx + new)
    st["kv_tiles"][1:] = ((ctx + new + TILE - 1) // TILE).cumsum(0)
    row = torch.arange(len(st["slots"]), device="cuda")
    r = torch.searchsorted(st["cu_new"][1:].long(), row, right=True).clamp(max=n - 1)
    token = ctx[r] + row - st["cu_new"][r]
    there = row < st["cu_new"][-1]
    entry = st["tables"][r, torch.where(there, token // page, 0)]
    st["slots"].copy_(torch.where(there, entry * page + token % page, -1))
    st["result"][0] = 0
    st["result"][1], st["result"][2], st["result"][3] = need.sum(), st["cu_new"][-1], st["kv_tiles"][-1]
    return [st[k] for k in ("tables", "slots", "cu_new", "kv_lens", "kv_tiles", "result")]


def _append(st):
    heads, page = st["case"]["kv_heads"], st["case"]["page"]
    there = st["slots"] >= 0
    slot = st["slots"][there].long()
    for part, (name, tab) in enumerate((("k", "k_tab"), ("v", "v_tab"))):
        x = st["qkv"][there, (1 + part) * heads:(2 + part) * heads]
        blocks = _encode(x.reshape(-1, GROUP), st[tab]).view(-1, heads, BLOCK_BYTES)
        st[name][slot // page, :, slot % page] = blocks
    return st["k"], st["v"]


def _request_blocks(st, name):
    """Blocks of all requests' tokens, [sum of kv][heads][64]."""
    page = st["case"]["page"]
    rows = []
    for r, kv in enumerate(st["kv_host"]):
        token = torch.arange(kv, device="cuda")
        rows.append(st["tables"][r, token // page].long() * page + token % page)
    slot = torch.cat(rows)
    return st[name][slot // page, :, slot % page]


def _attn(st):
    heads, g, causal = st["case"]["kv_heads"], st["case"]["q_per_kv"], st["case"]["causal"]
    k, v = (_decode(_request_blocks(st, name).reshape(-1, BLOCK_BYTES), st[tab]).view(-1, heads, GROUP) for name, tab in (("k", "k_tab"), ("v", "v_tab")))
    out, lse = torch.zeros_like(st["q"]), torch.full(st["q"].shape[:2], -math.inf, device="cuda")
    q0 = t0 = 0
    for new, kv in zip(st["new_host"], st["kv_host"]):
        for a in range(0, new, 512):
            b = min(a + 512, new)
            q = st["q"][q0 + a:q0 + b].float().view(b - a, heads, g, GROUP)
            s = torch.einsum("ihgd,thd->hgit", q, k[t0:t0 + kv]) * st["scale"]
            if causal:
                s.masked_fill_(torch.arange(kv, device="cuda") > kv - new + torch.arange(a, b, device="cuda")[:, None], -math.inf)
            top = s.amax(3, keepdim=True)
            p = (s - top).exp()
            total = p.sum(3, keepdim=True)
            o = torch.einsum("hgit,thd->ihgd", p, v[t0:t0 + kv]) / total.permute(2, 0, 1, 3)
            out[q0 + a:q0 + b] = o.reshape(b - a, heads * g, GROUP).half()
            lse[q0 + a:q0 + b] = (top + total.log())[..., 0].permute(2, 0, 1).reshape(b - a, heads * g)
        q0 += new
        t0 += kv
    return out, lse


def run(st):
    case = st["case"]
    if not own:
        return {"plan": _plan, "append": _append, "attn": _attn}[case["op"]](st)
    from paper_2505_06901_b200 import binding as B

    if case["op"] == "plan":
        B.ecco_paged_plan(case["page"], st["pages"], len(st["new"]), st["ctx"], st["new"], st["free"], len(st["free"]), st["tables"], st["stride"],
                          st["slots"], len(st["slots"]), st["cu_new"], st["kv_lens"], st["kv_tiles"], st["result"])
        return [st[k] for k in ("tables", "slots", "cu_new", "kv_lens", "kv_tiles", "result")]
    if case["op"] == "append":
        heads, row = case["kv_heads"], st["qkv"].data_ptr()
        B.ecco_paged_append(st["cache"], row + heads * GROUP * 2, row + 2 * heads * GROUP * 2, 3 * heads * GROUP, st["slots"], case["tokens"])
        return st["k"], st["v"]
    B.ecco_paged_attn(st["cache"], st["batch"], case["q_per_kv"], st["q"], st["q"].shape[1] * GROUP, st["scale"], B.ATTN_CAUSAL if case["causal"] else 0,
                      st["out"], st["lse"], st["ws"], st["ws_bytes"])
    return st["out"], st["lse"]


# ------------------------------------------------------------------ the definition, in 64 bits
def _exact_values(blocks, kind):
    """Bit by bit: a codeword of L bits is the symbol whose canonical number it is."""
    if len(blocks) > 131072:
        return torch.cat([_exact_values(part, kind) for part in blocks.split(131072)])
    t, dev, n = _tables(kind), blocks.device, len(blocks)
    to = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)  # noqa: E731

    def canonical(length, longest):
        length = np.asarray(length).reshape(-1, length.shape[-1])
        count = np.stack([(length == L).sum(1) for L in range(longest + 1)], 1)
        count[:, 0] = 0
        first, before = np.zeros_like(count), np.cumsum(count, 1) - count
        for L in range(1, longest + 1):
            first[:, L] = (first[:, L - 1] + count[:, L - 1]) * 2
        return to(count), to(first), to(before), to(np.argsort(length, axis=1, kind="stable"))

    bits = (blocks[:, :, None] >> torch.arange(8, dtype=torch.uint8, device=dev) & 1).view(n, BLOCK_BITS)
    bits = torch.cat([bits, torch.zeros((n, 16), dtype=torch.uint8, device=dev)], 1)

    def symbol(pos, row, tables, longest):
        count, first, before, order = (x[row] for x in tables)
        code, found, size = torch.zeros_like(pos), torch.full_like(pos, -1), torch.zeros_like(pos)
        for L in range(1, longest + 1):
            code = code * 2 + bits.gather(1, (pos + L - 1).clamp(max=BLOCK_BITS + 15)[:, None])[:, 0]
            at = code - first[:, L]
            hit = (found < 0) & (at >= 0) & (at < count[:, L])
            found = torch.where(hit, order.gather(1, (before[:, L] + at).clamp(0, order.shape[1] - 1)[:, None])[:, 0], found)
            size = torch.where(hit, L, size)
        return found, size

    def number(first, count):
        return (bits[:, first:first + count].long() << torch.arange(count, device=dev)).sum(1)

    def e4m3(byte):
        exp, man = (byte >> 3 & 15).double(), (byte & 7).double()
        size = torch.where(exp == 0, man / 8 * 2.0 ** -6, (1 + man / 8) * torch.exp2(exp - 7))
        return torch.where(byte >= 128, -size, size) * 2.0 ** EXPONENT

    def held(x):                                           # the format's one rounding: to fp16
        return x.clamp(-HALF_MAX, HALF_MAX).half().double()

    scale = e4m3(number(0, 8))
    one = torch.zeros(n, dtype=torch.int64, device=dev)
    kp, size = symbol(one + 10, one, canonical(t["kp_length"][None], 12), 12)
    pos, books = 10 + size, canonical(t["length"], 8)
    values = torch.zeros((n, GROUP), dtype=torch.float64, device=dev)
    whole, book = torch.ones(n, dtype=torch.bool, device=dev), kp * CODEBOOKS + number(8, 2)
    patterns = to(t["patterns"]).double()
    for i in range(GROUP):
        sym, size = symbol(pos, book, books, 8)
        whole &= pos + size <= BLOCK_BITS
        values[:, i] = torch.where(whole, torch.where(sym == 15, held(scale), held(patterns[kp, sym.clamp(max=14)] * scale.abs())), 0.0)
        pos = torch.where(whole, pos + size, pos)
    for j in range(16):
        field = number(BLOCK_BITS - 15 * (j + 1), 15)
        here = whole & (BLOCK_BITS - pos >= 15 * (j + 1))
        r = here.nonzero()[:, 0]
        values[r, field[r] & 127] = held(e4m3(field[r] >> 7))
    return values


def exact(case, seed):
    if case["op"] != "attn":
        return None                                        # whole numbers and bytes
    st = prepare(case, seed)
    new, ctx = _lengths(case)
    kv, _ = _seen(new, ctx, case["causal"])
    heads, g, page = case["kv_heads"], case["q_per_kv"], case["page"]
    if int(kv.sum()) * heads > 3_000_000:
        return None
    outs, lses, q0 = [], [], 0
    for r in range(len(new)):
        n, length = int(new[r]), int(kv[r])
        pages = st["tables"][r, :-(-length // page)].long()
        k, v = (_exact_values(st[name][pages].permute(0, 2, 1, 3).reshape(-1, heads, BLOCK_BYTES)[:length].reshape(-1, BLOCK_BYTES), name)
                .view(length, heads, GROUP) for name in ("k", "v"))
        q = st["q"][q0:q0 + n].double()
        q0 += n
        out = torch.empty((n, heads * g, GROUP), dtype=torch.float64, device="cuda")
        lse = torch.empty((n, heads * g), dtype=torch.float64, device="cuda")
        for h in range(heads * g):
            s = q[:, h] @ k[:, h // g].T * st["scale"]
            if case["causal"]:
                s = torch.where(torch.ones_like(s).tril(length - n) > 0, s, -math.inf)
            lse[:, h] = s.logsumexp(1)
            out[:, h] = (s - lse[:, h, None]).exp() @ v[:, h // g]
        outs.append(out)
        lses.append(lse)
    return torch.cat(outs), torch.cat(lses)
