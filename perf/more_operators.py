"""Rotary positions, and the paged cache in 8 bits: new tokens into it with their positions on the way, attention out of it.

A case is a dict of plain values; `op` says which operator one pass goes through:

  rope     ecco_rope_apply: rows of q and k of one projection turned by their positions
  append   ecco_paged8_append: K (turned by its position) and V rows of new tokens, as E4M3 numbers under a power of two for each block of
           tokens and head, into the slots of their tokens
  attn     ecco_paged8_attn: each request's new tokens attend to the request's pages (causal: the new tokens are the cache's
           last; otherwise, as with an encoder's states, every new token sees all of it)

The cache: a pool of pages [page][KV head][place][128] of E4M3 bytes, and an E8M0 byte (a power of two) for each block of min(16, page
size) places of a page and head: the smallest of 2^-15 .. 2^7 under which the block's largest value is at most 448.  A block that gets
more tokens keeps its power of two, or takes a larger one; then the values that it has are rounded again.  A token at a block's first
place begins the block anew.  K are N(0,1) with four channels of every head ten times as large, V are N(0,1).
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False                 # true: the framework's operators instead of the plain forms

GROUP = 128                 # values to a head
BLOCK = 16                  # places to a power of two
TILE = 32                   # tokens to a tile of a batch's kv_tiles
LOWEST, HIGHEST, BIAS = -15, 7, 127


def listed():
    return [
        # q and k rows of a decode step of 32 sequences, 32 + 8 heads: once per layer and token.
        {"name": "rope_step", "op": "rope", "tokens": 32, "heads": 40, "rot": 128, "pairs": "halves", "scaling": "none", "far": 4096, "prompt": False},
        # A batch of odd size, a third of its rows V that nobody turns; only half of each head has positions, in neighbouring pairs.
        {"name": "rope_part", "op": "rope", "tokens": 777, "heads": 24, "rot": 64, "pairs": "neighbours", "scaling": "none", "far": 16384, "prompt": False},
        # A piece of a long prompt, far into a context that frequencies by bands have made longer: the largest.
        {"name": "rope_prompt", "op": "rope", "tokens": 8192, "heads": 40, "rot": 128, "pairs": "halves", "scaling": "bands", "far": 131072, "prompt": True},
        # K and V rows of one new token for 32 sequences with eight KV heads: once per layer and decode step.
        {"name": "append_step", "op": "append", "requests": 32, "new": "1-1", "ctx": "0-79", "skipped": 0, "kv_heads": 8, "page": 16, "rot": 128, "pairs": "halves",
         "len_seed": 1},
        # Drafted tokens and pieces of prompts, padded to a fixed size for a captured graph; part of the head has positions.
        {"name": "append_padded", "op": "append", "requests": 24, "new": "1-8+1-8+20-90", "ctx": "0-90", "skipped": 90, "kv_heads": 8, "page": 64, "rot": 64,
         "pairs": "neighbours", "len_seed": 2},
        # The prompts of eight sequences of 512 tokens, 32 heads.
        {"name": "append_prompts", "op": "append", "requests": 8, "new": "512-512", "ctx": "0-0", "skipped": 0, "kv_heads": 32, "page": 64, "rot": 128,
         "pairs": "halves", "len_seed": 3},
        # Early in two conversations: the smallest decode step.
        {"name": "attn_step_short", "op": "attn", "requests": 2, "new": "1-1", "ctx": "770-783", "kv_heads": 8, "q_per_kv": 4, "page": 16, "causal": True,
         "len_seed": 4},
        # Decode step without grouped heads, eight sequences near 4096 tokens.
        {"name": "attn_step_mha", "op": "attn", "requests": 8, "new": "1-1", "ctx": "4000-4095", "kv_heads": 32, "q_per_kv": 1, "page": 64, "causal": True,
         "len_seed": 5},
        # Decode step of 32 requests of all lengths up to 16384: the largest cache.
        {"name": "attn_step_ragged", "op": "attn", "requests": 32, "new": "1-1", "ctx": "1-16383", "kv_heads": 8, "q_per_kv": 8, "page": 32, "causal": True,
         "len_seed": 6},
        # Four to eight drafted tokens of each of sixteen requests on their way through the target.
        {"name": "attn_drafts", "op": "attn", "requests": 16, "new": "4-8", "ctx": "10-4095", "kv_heads": 8, "q_per_kv": 4, "page": 16, "causal": True,
         "len_seed": 7},
        # A server's mixed batch: mostly single tokens, some pieces of prompts.
        {"name": "attn_mixed", "op": "attn", "requests": 24, "new": "1-1+1-1+1-1+1-500", "ctx": "0-3000", "kv_heads": 8, "q_per_kv": 4, "page": 16,
         "causal": True, "len_seed": 8},
        # The last 2048 tokens of each of two prompts of about 8000: the most arithmetic.
        {"name": "attn_chunk_long", "op": "attn", "requests": 2, "new": "2048-2048", "ctx": "5900-6144", "kv_heads": 8, "q_per_kv": 4, "page": 64,
         "causal": True, "len_seed": 9},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "attn", "attn", "attn"])
    page = rng.choice([1, 8, 16, 16, 32, 64, 128])
    turned = {"rot": rng.choice([16, 32, 64, 96, 128, 128, 128]), "pairs": rng.choice(["halves", "neighbours"])}
    if op == "rope":
        heads = rng.choice([1, 2, 5, 8, 12, 24, 40, 48])
        return {"op": op, "tokens": _log_int(rng, 1, 320_000 // heads), "heads": heads, **turned, "scaling": rng.choice(["none", "linear", "bands"]),
                "far": _log_int(rng, 16, 1 << 20), "prompt": rng.random() < 0.5}
    if op == "append":
        heads = rng.choice([1, 2, 4, 8, 8, 16, 32])
        requests = _log_int(rng, 1, 64)
        new = max(1, min(_log_int(rng, 1, 4096), 131_072 // (heads * requests)))
        return {"op": op, "requests": requests, "new": "%d-%d" % (rng.choice([1, 1, new]), new), "ctx": "0-%d" % _log_int(rng, 1, 100),
                "skipped": rng.choice([0, rng.randint(0, 100)]), "kv_heads": heads, "page": page, **turned, "len_seed": rng.randrange(1 << 30)}
    heads = rng.choice([1, 2, 4, 8, 8, 12, 32])
    q_per_kv = rng.choice([1, 1, 2, 3, 4, 4, 5, 8, 8])
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
    return {"op": op, "requests": requests, "new": new, "ctx": "%d-%d" % (rng.randint(1, ctx), ctx), "kv_heads": heads, "q_per_kv": q_per_kv, "page": page,
            "causal": rng.random() < 0.8, "len_seed": rng.randrange(1 << 30)}


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
    if case["op"] == "rope":
        n = case["tokens"] * case["heads"] * GROUP
        return {"bytes": 4 * n + 4 * case["tokens"], "flops": case["tokens"] * case["heads"] * case["rot"] * 3}
    new, ctx = _lengths(case)
    heads = case["kv_heads"]
    if case["op"] == "append":
        place = min(BLOCK, case["page"])
        blocks, begun = -(-(ctx + new) // place) - ctx // place, ctx % place > 0
        rows = int(new.sum())
        return {"bytes": int(2 * rows * heads * (2 * GROUP + GROUP) + 2 * heads * (blocks.sum() + begun.sum()) + 8 * rows + 4 * case["skipped"]),
                "flops": rows * heads * case["rot"] * 3}
    kv, pairs = _seen(new, ctx, case["causal"])
    q_heads = heads * case["q_per_kv"]
    pages, blocks = -(-kv // case["page"]), -(-kv // min(BLOCK, case["page"]))
    return {"bytes": int(2 * GROUP * kv.sum() * heads + 2 * blocks.sum() * heads + new.sum() * q_heads * (2 * GROUP * 2 + 4) + 4 * pages.sum() + 8 * len(new)),
            "flops": 4 * GROUP * q_heads * pairs}


# ------------------------------------------------------------------ what a program has in hand
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def _rows(kind, shape, gen):
    x = torch.randn(shape, generator=gen, device="cuda")
    if kind == "k":
        x[..., 3::32] *= 10
    return x.half()


def _frequencies(case):
    """Radians per position of each pair; a context 8 times as long as it was learnt (8192) by all or by the slow pairs alone."""
    f = 10000.0 ** (-np.arange(0, case["rot"], 2) / case["rot"])
    scaling = case.get("scaling", "none")
    if scaling == "linear":
        f = f / 8
    elif scaling == "bands":
        whole = np.clip((8192 * f / (2 * math.pi) - 1) / 3, 0, 1)       # four turns and more: as they are; less than one: all the slower
        f = f * (whole + (1 - whole) / 8)
    return f


def _turned(case, st):
    st["frequencies"] = torch.from_numpy(_frequencies(case)).cuda()
    if own:
        from paper_2505_06901_b200 import binding as B

        st["rope"] = B.ecco_rope_init(case["rot"], _frequencies(case), flags=B.ROPE_NEIGHBOURS if case["pairs"] == "neighbours" else 0)


def _cache(st, case, pages, gen):
    heads, page = case["kv_heads"], case["page"]
    places, blocks = min(BLOCK, page), max(1, page // BLOCK)
    for kind in ("k", "v"):
        pool = torch.empty((pages, heads, page, GROUP), dtype=torch.uint8, device="cuda")
        scales = torch.empty((pages, heads, blocks), dtype=torch.uint8, device="cuda")
        step = max(1, (1 << 26) // (heads * page * GROUP))
        for a in range(0, pages, step):
            x = _rows(kind, pool[a:a + step].shape, gen).view(-1, heads, blocks, places, GROUP)
            e = _power_of(x.float().abs().amax((3, 4)))
            pool[a:a + step] = _to_e4m3(x.float(), e[..., None, None]).view(-1, heads, page, GROUP)
            scales[a:a + step] = (e + BIAS).to(torch.uint8)
        st[kind], st[kind + "_scales"] = pool, scales
    if own:
        from paper_2505_06901_b200 import binding as B

        st["cache"] = B.paged8_cache(st["k"], st["v"], st["k_scales"], st["v_scales"], pages, heads, page)


def _tables(st, kv, page, spare, gen):
    held = -(-kv // page)
    pages = int(held.sum()) + spare
    st["stride"] = int(held.max()) + 1
    st["tables"] = torch.full((len(kv), st["stride"]), -1, dtype=torch.int32, device="cuda")
    st["tables"][torch.arange(st["stride"], device="cuda") < _ints(held)[:, None]] = torch.randperm(pages, generator=gen, device="cuda").int()[:int(held.sum())]
    return pages


def prepare(case, seed):
    gen = _generator(seed)
    st = {"case": case}
    if case["op"] == "rope":
        tokens, heads = case["tokens"], case["heads"]
        if case["prompt"]:
            positions = torch.arange(tokens, device="cuda") + max(0, case["far"] - tokens)
        else:
            positions = torch.randint(case["far"], (tokens,), generator=gen, device="cuda")
        # rows of one projection: the heads that are turned, and V of a quarter as many
        st.update(positions=positions.int(), qkv=torch.randn((tokens, heads + -(-heads // 4), GROUP), generator=gen, device="cuda").half(),
                  out=torch.empty((tokens, heads, GROUP), dtype=torch.float16, device="cuda"))
        _turned(case, st)
        return st
    new, ctx = _lengths(case)
    heads, page = case["kv_heads"], case["page"]
    if case["op"] == "append":
        _cache(st, case, _tables(st, ctx + new, page, 2, gen), gen)
        rows = int(new.sum())
        r = np.repeat(np.arange(len(new)), new)
        token = np.arange(rows) - np.repeat(np.cumsum(new) - new, new) + ctx[r]
        slots = torch.full((rows + case["skipped"],), -1, dtype=torch.int32, device="cuda")
        slots[:rows] = st["tables"][_ints(r).long(), _ints(token // page).long()] * page + _ints(token % page)
        positions = torch.zeros_like(slots)
        positions[:rows] = _ints(token)
        # K and V as parts of the rows that one projection writes: queries (as many heads again), keys, values
        qkv = torch.zeros((len(slots), 3 * heads, GROUP), dtype=torch.float16, device="cuda")
        qkv[:, heads:2 * heads], qkv[:, 2 * heads:] = _rows("k", (len(slots), heads, GROUP), gen), _rows("v", (len(slots), heads, GROUP), gen)
        st.update(qkv=qkv, slots=slots, positions=positions)
        _turned(case, st)
        return st
    kv, _ = _seen(new, ctx, case["causal"])
    _cache(st, case, _tables(st, kv, page, 7, gen), gen)
    q_per_kv, tokens = case["q_per_kv"], int(new.sum())
    tiles = np.concatenate([[0], np.cumsum(-(-kv // TILE))])
    st.update(kv_lens=_ints(kv), kv_tiles=_ints(tiles), cu_new=_ints(np.concatenate([[0], np.cumsum(new)])),
              q=torch.randn((tokens, heads * q_per_kv, GROUP), generator=gen, device="cuda").half(), new_host=new.tolist(), kv_host=kv.tolist(), scale=GROUP ** -0.5)
    if own:
        from paper_2505_06901_b200 import binding as B

        st["batch"] = B.paged_batch(st["tables"], st["stride"], st["cu_new"], st["kv_lens"], st["kv_tiles"], len(new), tokens, int(new.max()), int(kv.max()), int(tiles[-1]))
        st["ws_bytes"] = B.ecco_paged8_attn_workspace_bytes(st["cache"], st["batch"], q_per_kv)
        st["ws"] = torch.empty(st["ws_bytes"], dtype=torch.uint8, device="cuda")
        st["out"] = torch.empty((tokens, heads * q_per_kv, GROUP), dtype=torch.float16, device="cuda")
        st["lse"] = torch.empty((tokens, heads * q_per_kv), device="cuda")
    return st


# ------------------------------------------------------------------ plain forms
def _power_of(top):
    """The smallest e with top <= 448 * 2^e = 0.875 * 2^(e + 9), in its range."""
    m, k = torch.frexp(top)
    return torch.where(top > 0, k - 9 + (m > 0.875), LOWEST).clamp(LOWEST, HIGHEST)


def _to_e4m3(x, e):
    return (x * torch.exp2(-e.float())).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _turn(x, positions, frequencies, pairs):
    """fp16 [tokens][heads][128] turned by positions: angles in 64 bits, the rest in 32."""
    angle = positions.double()[:, None] * frequencies
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
    rot = 2 * frequencies.numel()
    y = x.float()
    first, second = (y[..., 0:rot:2], y[..., 1:rot:2]) if pairs == "neighbours" else (y[..., :rot // 2], y[..., rot // 2:rot])
    first, second = first * c - second * s, second * c + first * s
    part = torch.stack([first, second], -1).flatten(-2) if pairs == "neighbours" else torch.cat([first, second], -1)
    return torch.cat([part, y[..., rot:]], -1).half()


def _rope(st):
    case = st["case"]
    return _turn(st["qkv"][:, :case["heads"]], st["positions"], st["frequencies"], case["pairs"])


def _outputs(st):
    return [st[k].view(torch.float8_e4m3fn) for k in ("k", "v")] + [st[k].view(torch.float8_e8m0fnu) for k in ("k_scales", "v_scales")]


def _append(st):
    case = st["case"]
    heads, page = case["kv_heads"], case["page"]
    places = min(BLOCK, page)
    there = st["slots"] >= 0
    slot = st["slots"][there].long()
    qkv = st["qkv"][there]
    block, mine = torch.unique(slot // places, return_inverse=True)
    at, nth = block * places // page, block % (page // places)            # page, and block of the page
    begun = torch.full_like(block, page).scatter_reduce(0, mine, slot % places, "amin") > 0
    for kind, x in (("k", _turn(qkv[:, heads:2 * heads], st["positions"][there], st["frequencies"], case["pairs"])), ("v", qkv[:, 2 * heads:])):
        top = torch.zeros((len(block), heads), device="cuda").index_reduce(0, mine, x.float().abs().amax(2), "amax")
        pool, scales = st[kind], st[kind + "_scales"]
        before = scales[at, :, nth].int() - BIAS
        e = _power_of(top)
        e = torch.where(begun[:, None], torch.maximum(e, before), e)
        blocks = pool.view(len(pool), heads, -1, places, GROUP)
        held = blocks[at, :, nth]
        again = _to_e4m3(held.view(torch.float8_e4m3fn).float() * torch.exp2(before.float())[..., None, None], e[..., None, None])
        blocks[at, :, nth] = torch.where(begun[:, None, None, None], again, held)
        pool[slot // page, :, slot % page] = _to_e4m3(x.float(), e[mine][..., None])
        scales[at, :, nth] = (e + BIAS).to(torch.uint8)
    return _outputs(st)


def _request_values(st, kind):
    """Values of all requests' tokens, fp32 [sum of kv][heads][128]."""
    page = st["case"]["page"]
    slot = torch.cat([st["tables"][r, t // page].long() * page + t % page for r, t in enumerate(torch.arange(kv, device="cuda") for kv in st["kv_host"])])
    at, place = slot // page, slot % page
    scale = torch.exp2(st[kind + "_scales"][at, :, place // BLOCK].float() - BIAS)
    return st[kind][at, :, place].view(torch.float8_e4m3fn).float() * scale[..., None]


def _attn(st):
    heads, g, causal = st["case"]["kv_heads"], st["case"]["q_per_kv"], st["case"]["causal"]
    k, v = _request_values(st, "k"), _request_values(st, "v")
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


# ------------------------------------------------------------------ one pass
def run(st):
    case = st["case"]
    if not own:
        return {"rope": _rope, "append": _append, "attn": _attn}[case["op"]](st)
    from paper_2505_06901_b200 import binding as B

    if case["op"] == "rope":
        B.ecco_rope_apply(st["rope"], st["positions"], case["tokens"], case["heads"], st["qkv"], st["qkv"].shape[1] * GROUP, st["out"], case["heads"] * GROUP)
        return st["out"]
    if case["op"] == "append":
        heads, row = case["kv_heads"], st["qkv"].data_ptr()
        B.ecco_paged8_append(st["cache"], st["rope"], st["positions"], row + heads * GROUP * 2, row + 2 * heads * GROUP * 2, 3 * heads * GROUP, st["slots"],
                             len(st["slots"]))
        return _outputs(st)
    B.ecco_paged8_attn(st["cache"], st["batch"], case["q_per_kv"], st["q"], st["q"].shape[1] * GROUP, st["scale"], B.ATTN_CAUSAL if case["causal"] else 0,
                       st["out"], st["lse"], st["ws"], st["ws_bytes"])
    return st["out"], st["lse"]


# ------------------------------------------------------------------ the definition, in 64 bits
def _exact_turn(x, positions, case):
    """Pair by pair, as complex numbers times e^(i angle); the whole turns are taken off before the angle is formed."""
    rot = case["rot"]
    turns = torch.from_numpy(_frequencies(case) / (2 * math.pi)).cuda()
    coarse = torch.round(turns * 2 ** 30) / 2 ** 30                         # times a position below 2^21 exact
    p = positions.double()[:, None]
    angle = 2 * math.pi * ((p * coarse).remainder(1.0) + p * (turns - coarse))
    y = x.double()
    first = torch.arange(0, rot, 2, device="cuda") if case["pairs"] == "neighbours" else torch.arange(rot // 2, device="cuda")
    second = first + (1 if case["pairs"] == "neighbours" else rot // 2)
    z = torch.complex(y[..., first], y[..., second]) * torch.polar(torch.ones_like(angle), angle)[:, None]
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _nearest_e4m3(y):
    """The number of three mantissa bits nearest to y, ties to even, as an fp64 number."""
    y = y.clamp(-448, 448)
    step = torch.exp2((torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -9)))).clamp(min=-6) - 3)
    return torch.round(y / step) * step


def _e4m3_value(byte):
    exp, man = (byte >> 3 & 15).double(), (byte & 7).double()
    size = torch.where(exp == 0, man / 8 * 2.0 ** -6, (1 + man / 8) * torch.exp2(exp - 7))
    return torch.where(byte >= 128, -size, size)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rope":
        return _exact_turn(st["qkv"][:, :case["heads"]], st["positions"], case)
    heads, page = case["kv_heads"], case["page"]
    new, ctx = _lengths(case)
    places = min(BLOCK, page)
    if case["op"] == "append":
        rows = int(new.sum())
        qkv = st["qkv"][:rows]
        pools, scales = [], []
        slot = st["slots"][:rows].long()
        for kind, x in (("k", _exact_turn(qkv[:, heads:2 * heads], st["positions"][:rows], case).half().double()), ("v", qkv[:, 2 * heads:].double())):
            value = _e4m3_value(st[kind].long()).permute(0, 2, 1, 3).reshape(-1, heads, GROUP)          # [slot][head]
            power = st[kind + "_scales"].long().permute(0, 2, 1).reshape(-1, heads) - BIAS             # [block][head]
            block = slot // places
            top = torch.zeros(power.shape, dtype=torch.float64, device="cuda").index_reduce(0, block, x.abs().amax(2), "amax")
            touched, anew = torch.zeros(len(power), dtype=torch.bool, device="cuda"), torch.zeros(len(power), dtype=torch.bool, device="cuda")
            touched[block], anew[block[slot % places == 0]] = True, True
            need = torch.full_like(power, LOWEST)
            for e in range(HIGHEST, LOWEST - 1, -1):                      # the smallest that does
                need = torch.where(top <= 448.0 * 2.0 ** e, e, need) if e < HIGHEST else torch.full_like(power, e)
            after = torch.where(touched[:, None], torch.where(anew[:, None], need, torch.maximum(need, power)), power)
            shrink = torch.exp2((power - after).double()).repeat_interleave(places, 0)[..., None]
            keep = (touched & ~anew)[:, None].expand_as(power).repeat_interleave(places, 0)[..., None]
            value = torch.where(keep, _nearest_e4m3(value * shrink), value)
            value[slot] = _nearest_e4m3(x * torch.exp2(-after[block].double())[..., None])
            pools.append(value.view(-1, page, heads, GROUP).permute(0, 2, 1, 3).contiguous())
            scales.append(torch.exp2(after.double()).view(-1, page // places, heads).permute(0, 2, 1).contiguous())
        return pools + scales
    kv, _ = _seen(new, ctx, case["causal"])
    g = case["q_per_kv"]
    if int(kv.sum()) * heads > 3_000_000:
        return None
    outs, lses, q0 = [], [], 0
    for r in range(len(new)):
        n, length = int(new[r]), int(kv[r])
        pages = st["tables"][r, :-(-length // page)].long()
        k, v = ((_e4m3_value(st[name][pages].long()).view(len(pages), heads, -1, places, GROUP) * torch.exp2(st[name + "_scales"][pages].double() - BIAS)[..., None, None])
                .view(len(pages), heads, page, GROUP).permute(0, 2, 1, 3).reshape(-1, heads, GROUP)[:length] for name in ("k", "v"))
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
