"""The paged KV cache: ecco_paged_plan, ecco_paged_append, ecco_paged_attn.

Reference: plans in plain Python, blocks by the oracle's encoder, attention in 64 bits over what the oracle's decoder makes of the
blocks.  Tolerances of the attention, per output, from the kernels' roundings:
  scores: 128 products, exact in fp32, added on the tensor cores, which cut off: eps_s = 128 * 2^-23 * scale * max_t sum |q k|, and one
          rounding each of scale * log2(e), of the product with it and of the difference to the maximum: 2^-22 * |s|;
  weights: fp16, half a step 2^-11 of each; exp2 2^-22.  They stand at 2^7 times what they are relative to a maximum that is at most the
          row's own, so below fp16's normal range half a step is 2^-25 / 2^7 = 2^-32 of the largest weight or less;
  sums over n tokens on the tensor cores, sixteen a step: (n / 16 + 32) * 2^-23;
  the output's own rounding: 2^-11 of it, or 2^-25.
  |out - ref| <= 2^-11 |ref| + (2^-11 + 2 e_s + (n / 16 + 32) 2^-23) sum p |v| + 2^-32 sum |v| + 2^-25, e_s = eps_s + 2^-22 max |s| + 2^-22
  |lse - ref| <= e_s + (n / 16 + 32) 2^-23 + 2^-22 |ref| + 2^-20.
"""
import ctypes
import math

import numpy as np
import pytest

from helpers import lib_meta_from_oracle

torch = pytest.importorskip("torch")


@pytest.fixture(scope="session")
def B():
    from paper_2505_06901_b200 import binding as b

    b.lib()
    return b


@pytest.fixture(scope="session")
def dev():
    if not torch.cuda.is_available():
        pytest.fail("the gpu tests need a CUDA device")
    return "cuda"


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------ refusals, on the CPU
def test_argument_errors_without_a_gpu(B):
    L, INV, ALIGN = B.lib(), B.ERR_INVALID_ARG, B.ERR_ALIGNMENT

    def plan(page=16, pages=8, n_req=2, ctx=64, new=64, free=64, n_free=4, tables=64, stride=4, slots=64, n_slots=9, cu=64, lens=64, tiles=64, result=64):
        return L.ecco_paged_plan(page, pages, n_req, ctx, new, free, n_free, tables, stride, slots, n_slots, cu, lens, tiles, result, None)

    for bad in (dict(page=0), dict(page=12), dict(page=8192), dict(pages=0), dict(page=4096, pages=1 << 19), dict(n_req=-1), dict(n_req=65536), dict(n_free=-1),
                dict(stride=-1), dict(n_slots=-1), dict(ctx=None), dict(new=None), dict(free=None), dict(tables=None), dict(slots=None), dict(cu=None),
                dict(lens=None), dict(tiles=None), dict(result=None)):
        assert plan(**bad) == INV, bad
    for name in ("ctx", "new", "free", "tables", "slots", "cu", "lens", "tiles", "result"):
        assert plan(**{name: 66}) == ALIGN, name
    assert plan(ctx=128) == INV and plan(new=128) == INV                       # the new lengths over the ones that they come from

    def cache(k_meta=64, v_meta=64, k=64, v=64, pages=8, heads=2, page=16):
        return B.PagedCache(k_meta, v_meta, k, v, pages, heads, page)

    def append(c=None, k=64, v=64, stride=256, slots=64, n=3):
        return L.ecco_paged_append(ctypes.byref(c or cache()), k, v, stride, slots, n, None)

    bad_caches = (dict(k_meta=None), dict(v_meta=None), dict(k=None), dict(v=None), dict(pages=0), dict(heads=0), dict(heads=65536), dict(page=3),
                  dict(page=4096, pages=1 << 19))
    assert append(n=0) == 0 and append(n=-1) == INV and L.ecco_paged_append(None, 64, 64, 256, 64, 3, None) == INV
    for bad in bad_caches:
        assert append(cache(**bad)) == INV, bad
    for bad in (dict(k=None), dict(v=None), dict(slots=None), dict(stride=248)):
        assert append(**bad) == INV, bad
    for bad in (dict(c=cache(k=80)), dict(c=cache(v=80)), dict(c=cache(k_meta=72)), dict(c=cache(v_meta=72)), dict(k=72), dict(v=72), dict(slots=66), dict(stride=257)):
        assert append(**bad) == ALIGN, bad

    def batch(tables=64, cu=64, lens=64, tiles=64, stride=4, n_req=2, tokens=3, new=2, kv=60, n_tiles=4):
        return B.PagedBatch(tables, cu, lens, tiles, stride, n_req, tokens, new, kv, n_tiles)

    def attn(c=None, b=None, g=2, q=64, stride=512, scale=0.1, flags=1, out=64, lse=64, ws=64, ws_bytes=1 << 30):
        return L.ecco_paged_attn(ctypes.byref(c or cache()), ctypes.byref(b or batch()), g, q, stride, ctypes.c_float(scale), flags, out, lse, ws, ws_bytes, None)

    assert attn(b=batch(n_req=0)) == 0 and attn(b=batch(tokens=0)) == 0                        # nothing to do
    for bad in bad_caches:
        assert attn(cache(**bad)) == INV, bad
    for bad in (dict(g=0), dict(g=17), dict(scale=math.nan), dict(scale=math.inf), dict(scale=3e38), dict(flags=2), dict(q=None), dict(out=None), dict(stride=504), dict(stride=1 << 38),
                dict(b=batch(tokens=1 << 26, kv=1 << 26)),
                dict(b=batch(tables=None)), dict(b=batch(cu=None)), dict(b=batch(lens=None)), dict(b=batch(tiles=None)), dict(b=batch(stride=-1)),
                dict(b=batch(n_req=65536)), dict(b=batch(tokens=-1)), dict(b=batch(new=-1)), dict(b=batch(kv=-1)), dict(b=batch(n_tiles=-1)),
                dict(b=batch(n_tiles=1 << 30))):
        assert attn(**bad) == INV, bad
    for bad in (dict(q=72), dict(out=72), dict(lse=66), dict(stride=513), dict(b=batch(tables=66)), dict(b=batch(cu=66)), dict(b=batch(lens=66)),
                dict(b=batch(tiles=66)), dict(c=cache(k=80))):
        assert attn(**bad) == ALIGN, bad
    assert attn(ws=128) == INV and attn(out=128) == INV and attn(q=128) == INV                  # two of the three are one
    need = lambda c, b, g: int(L.ecco_paged_attn_workspace_bytes(ctypes.byref(c), ctypes.byref(b), g))  # noqa: E731
    assert need(cache(), batch(), 2) >= 4 * 2 * 2 * 8192 and need(cache(), batch(), 0) == 0 and need(cache(), batch(n_tiles=-1), 2) == 0
    assert need(cache(heads=1), batch(), 2) < need(cache(heads=8), batch(), 2)


def test_every_bad_argument_is_refused_by_itself(B):
    """All other arguments are such that the call goes on to ask for the device, of which there is none: only the one that is bad can be
    what the call refuses."""
    if torch.cuda.is_available():
        pytest.skip("with a device the calls that are not refused would run on these addresses")
    L, INV, ALIGN, GONE = B.lib(), B.ERR_INVALID_ARG, B.ERR_ALIGNMENT, B.ERR_CUDA

    def check(call, names, invalid, null=()):
        base = {n: 4096 * (i + 1) for i, n in enumerate(names)}
        assert call(**base) == GONE
        for name in names:
            odd = call(**{**base, name: base[name] + 2})
            assert odd == ALIGN, name
            assert call(**{**base, name: None}) == (GONE if name in null else INV), name
        for bad in invalid:
            assert call(**{**base, **bad}) == INV, bad
        return base

    def plan(page=16, pages=8, n_req=2, n_free=4, stride=4, n_slots=9, **p):
        return L.ecco_paged_plan(page, pages, n_req, p["ctx"], p["new"], p["free"], n_free, p["tables"], stride, p["slots"], n_slots, p["cu"], p["lens"], p["tiles"],
                                 p["result"], None)

    pages = (dict(page=0), dict(page=-16), dict(page=12), dict(page=8192), dict(pages=0), dict(pages=-1), dict(page=4096, pages=1 << 19))
    p = check(plan, ("ctx", "new", "free", "tables", "slots", "cu", "lens", "tiles", "result"),
              pages + (dict(n_req=-1), dict(n_req=65536), dict(n_free=-1), dict(stride=-1), dict(n_slots=-1)))
    assert plan(**p | {"lens": p["ctx"]}) == INV and plan(**p | {"lens": p["new"]}) == INV           # the new lengths over the ones that they come from
    for largest in (dict(page=4096, pages=(1 << 19) - 1), dict(page=1, pages=2**31 - 1), dict(n_req=65535), dict(n_free=0, free=None), dict(n_slots=0, slots=None),
                    dict(stride=0, tables=None), dict(n_req=0, ctx=None, new=None, tables=None, lens=None)):
        assert plan(**p | largest) == GONE, largest

    def cache(k_meta, v_meta, k, v, heads=2, page=16, pages=8):
        return ctypes.byref(B.PagedCache(k_meta, v_meta, k, v, pages, heads, page))

    pools = ("k_meta", "v_meta", "k", "v")
    caches = pages + (dict(heads=0), dict(heads=-1), dict(heads=65536, stride=1 << 30))

    def append(kx, vx, slots, stride=256, n=3, **c):
        return L.ecco_paged_append(cache(**c), kx, vx, stride, slots, n, None)

    p = check(append, pools + ("kx", "vx", "slots"), caches + (dict(stride=248), dict(stride=-256), dict(n=-1)))
    assert append(**p | {"stride": 260}) == ALIGN and append(**p | {"n": 0}) == 0
    for largest in (dict(heads=65535, stride=65535 * 128), dict(n=2**31 - 1), dict(stride=1 << 50)):
        assert append(**p | largest) == GONE, largest
    for name in ("k", "v"):                                # pools: 32 bytes; metadata and rows: 16
        assert append(**p | {name: p[name] + 16}) == ALIGN
    for name in ("k_meta", "v_meta", "kx", "vx"):
        assert append(**p | {name: p[name] + 8}) == ALIGN and append(**p | {name: p[name] + 16}) == GONE, name

    def attn(tables, cu, lens, tiles, q, out, lse, ws, t_stride=4, n_req=2, tokens=3, new=2, kv=60, n_tiles=4, g=2, stride=512, scale=0.1, flags=1,
             ws_bytes=1 << 30, **c):
        b = B.PagedBatch(tables, cu, lens, tiles, t_stride, n_req, tokens, new, kv, n_tiles)
        return L.ecco_paged_attn(cache(**c), ctypes.byref(b), g, q, stride, ctypes.c_float(scale), flags, out, lse, ws, ws_bytes, None)

    # a workspace that is missing, misaligned or too small is found when the device is known
    arrays = ("tables", "cu", "lens", "tiles", "q", "out", "lse")
    p = check(lambda **a: attn(ws=1 << 20, **a), pools + arrays, caches + (
        dict(g=0), dict(g=-1), dict(g=17, stride=1 << 20), dict(scale=math.nan), dict(scale=math.inf), dict(scale=-math.inf), dict(scale=3e38), dict(flags=2), dict(flags=3), dict(flags=1 << 31),
        dict(stride=504), dict(stride=-512), dict(stride=1 << 38), dict(t_stride=-1), dict(n_req=-1), dict(n_req=65536), dict(tokens=-1), dict(new=-1), dict(kv=-1),
        dict(n_tiles=-1), dict(n_tiles=1 << 25, heads=64, stride=1 << 20), dict(n_tiles=1 << 26, heads=1), dict(heads=4096, g=16, stride=1 << 30), dict(tokens=1 << 29),
        dict(tokens=1 << 26, kv=1 << 26)), null=("lse",))
    p["ws"] = 1 << 20
    for name in ("q", "out"):
        assert attn(**p | {name: p[name] + 8}) == ALIGN, name
    assert attn(**p | {"stride": 516}) == ALIGN
    for a, b in (("out", "q"), ("out", "ws"), ("q", "ws")):
        assert attn(**p | {a: p[b]}) == INV, (a, b)
    for fine in (dict(g=1), dict(g=16, stride=4096), dict(scale=0.0), dict(scale=-2.0), dict(scale=2e38), dict(flags=0), dict(t_stride=0, tables=None), dict(n_req=65535),
                 dict(stride=(1 << 38) - 8), dict(new=0), dict(kv=0), dict(n_tiles=0), dict(tokens=1 << 20, kv=1 << 20), dict(n_tiles=1 << 20)):
        assert attn(**p | fine) == GONE, fine
    assert attn(**p | {"n_req": 0}) == 0 and attn(**p | {"tokens": 0}) == 0
    assert L.ecco_paged_append(None, 64, 128, 256, 192, 3, None) == INV
    assert L.ecco_paged_attn(None, ctypes.byref(B.PagedBatch(64, 128, 192, 256, 4, 2, 3, 2, 60, 4)), 2, 512, 512, ctypes.c_float(0.1), 1, 1024, None, 2048, 1 << 30, None) == INV
    c = cache(4096, 8192, 12288, 16384)
    assert L.ecco_paged_attn(c, None, 2, 512, 512, ctypes.c_float(0.1), 1, 1024, None, 2048, 1 << 30, None) == INV


# ------------------------------------------------------------------ plan
def plan_reference(page, n_pages, ctx, new, free, tables, n_slots):
    tables, slots, taken = tables.copy(), np.full(n_slots, -1, np.int32), 0
    cu, tiles, row = [0], [0], 0
    for r, (c, n) in enumerate(zip(ctx, new)):
        held, total = -(-c // page), -(-(c + n) // page)
        tables[r, held:total] = free[taken:taken + total - held]
        taken += total - held
        for t in range(c, c + n):
            e = tables[r, t // page]
            slots[row] = e * page + t % page if 0 <= e < n_pages else -1
            row += 1
        cu.append(row)
        tiles.append(tiles[-1] + -(-(c + n) // 32))
    return tables, slots, np.array(cu), np.asarray(ctx, dtype=np.int64) + new, np.array(tiles), np.array([0, taken, row, tiles[-1]])


def run_plan(B, page, n_pages, ctx, new, free, tables, n_slots):
    n = len(ctx)
    d_tables = ints(tables)
    out = [torch.full((k,), -7, dtype=torch.int32, device="cuda") for k in (n_slots, n + 1, n, n + 1, 4)]
    B.ecco_paged_plan(page, n_pages, n, ints(ctx), ints(new), ints(free), len(free), d_tables, tables.shape[1], out[0], n_slots, *out[1:])
    torch.cuda.synchronize()
    return [d_tables.cpu().numpy()] + [t.cpu().numpy() for t in out]


@pytest.mark.gpu
@pytest.mark.parametrize("n_req,page,max_ctx,max_new", [(1, 16, 0, 1), (1, 1, 0, 5000), (3, 16, 100, 40), (33, 64, 1000, 1), (1024, 16, 300, 9), (1025, 32, 50, 3),
                                                        (2500, 8, 70, 5), (7, 4096, 9000, 5000), (40, 128, 0, 128), (300, 16, 64, 0)])
def test_plan_matches_the_definition(B, dev, n_req, page, max_ctx, max_new):
    rng = np.random.default_rng([n_req, page])
    ctx, new = rng.integers(0, max_ctx + 1, n_req), rng.integers(0, max_new + 1, n_req)
    if n_req > 2:
        ctx[1] = ctx[1] // page * page                                         # a request that fills its last page
        new[2] = 0
    held, total = -(-ctx // page), -(-(ctx + new) // page)
    need = int((total - held).sum())
    n_pages = int(total.sum()) + 5
    ids = rng.permutation(n_pages).astype(np.int32)
    free, owned = ids[:need + 2], ids[need + 2:]
    tables = rng.integers(-5, 1 << 30, (n_req, int(total.max()) + 2)).astype(np.int32)          # what is not the request's is arbitrary
    at = 0
    for r in range(n_req):
        tables[r, :held[r]] = owned[at:at + held[r]]
        at += held[r]
    n_slots = int(new.sum()) + 13
    want = plan_reference(page, n_pages, ctx, new, free, tables, n_slots)
    got = run_plan(B, page, n_pages, ctx, new, free, tables, n_slots)
    for name, w, g in zip(("tables", "slots", "cu_new", "kv_lens", "kv_tiles", "result"), want, got):
        assert np.array_equal(w, g), name


@pytest.mark.gpu
def test_plan_without_requests_and_with_foreign_pages(B, dev):
    out = [torch.full((k,), -7, dtype=torch.int32, device="cuda") for k in (3, 1, 1, 4)]
    B.ecco_paged_plan(16, 4, 0, 0, 0, 0, 0, 0, 0, out[0], 3, out[1], 0, out[2], out[3])
    assert out[0].tolist() == [-1] * 3 and out[1].tolist() == [0] and out[2].tolist() == [0] and out[3].tolist() == [0, 0, 0, 0]
    # page ids that are not of the pool: the tokens get no slot
    tables = np.array([[-1, 9], [7, 4]], np.int32)
    got = run_plan(B, 4, 5, [2, 8], [3, 1], np.array([5, -3], np.int32), np.concatenate([tables, np.zeros((2, 1), np.int32)], 1), 6)
    assert got[1].tolist() == [-1] * 6 and got[0].tolist() == [[-1, 5, 0], [7, 4, -3]] and got[5].tolist() == [0, 2, 4, 4 - 2]


@pytest.mark.gpu
@pytest.mark.parametrize("what", ["negative ctx", "negative new", "row too long", "no page", "no slot", "too many", "too long"])
def test_plan_serves_all_or_none(B, dev, what):
    ctx, new, free, n_slots, stride = [5, 17, 0], [1, 20, 3], np.arange(10, 14, dtype=np.int32), 24, 3
    want = B.ERR_INVALID_ARG
    if what == "negative ctx":
        ctx[1] = -1
    elif what == "negative new":
        new[2] = -1
    elif what == "row too long":
        new[1], n_slots, free = 32, 100, np.arange(10, 20, dtype=np.int32)
    elif what == "no page":
        free, want = free[:1], B.ERR_WORKSPACE
    elif what == "no slot":
        n_slots, want = 23, B.ERR_WORKSPACE
    elif what in ("too many", "too long"):
        ctx, new, stride = ([0] * 3, [2**31 - 1] * 3, 1 << 20) if what == "too many" else ([2**31 - 5, 0, 0], [5, 0, 0], 1 << 20)
        # the table is not touched, so only its stride is large
        tables = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = [torch.full((k,), -7, dtype=torch.int32, device="cuda") for k in (5, 4, 3, 4, 4)]
        B.ecco_paged_plan(4096, 10, 3, ints(ctx), ints(new), ints(free), 4, tables, stride, out[0], 5, *out[1:])
        torch.cuda.synchronize()
        assert out[4].tolist() == [B.ERR_INVALID_ARG, 0, 0, 0] and out[0].tolist() == [-1] * 5
        return
    tables = np.arange(9, dtype=np.int32).reshape(3, 3)[:, :stride]
    got = run_plan(B, 16, 20, ctx, new, free, tables, n_slots)
    assert got[5].tolist() == [want, 0, 0, 0]
    assert np.array_equal(got[0], tables) and (got[1] == -1).all() and not got[2].any() and not got[3].any() and not got[4].any()


# ------------------------------------------------------------------ append
@pytest.mark.gpu
@pytest.mark.parametrize("tokens,heads,page,extra", [(1, 1, 1, 0), (5, 3, 16, 8), (33, 8, 64, 0), (700, 32, 16, 4096), (4096, 8, 128, 1024), (9001, 1, 32, 24)])
def test_append_writes_the_oracles_blocks_into_the_slots(B, dev, eo, kv_small, tokens, heads, page, extra):
    """Small calls and calls of many groups; K and V in the rows of a projection, padding tokens, slots outside of the pool."""
    rng = np.random.default_rng([tokens, heads])
    meta_k, src = kv_small["meta"], kv_small["k"].reshape(-1, 128)
    meta_v = eo.calibrate(kv_small["cal"].reshape(-1)[:128 * 512], S=16, H=4, seed=9, select=eo.SELECT_MINMAX)
    n_pages = -(-tokens // page) + 3
    slots = rng.permutation(n_pages * page)[:tokens].astype(np.int32)
    if tokens > 4:
        slots[[0, 3]] = -1
        slots[1], slots[2] = n_pages * page, 2**31 - 1
    rows = np.zeros((tokens, 2 * heads * 128 + extra), np.float16)
    pick = rng.integers(0, len(src), (2, tokens, heads))
    rows[:, :heads * 128] = src[pick[0]].reshape(tokens, -1)
    rows[:, -heads * 128:] = src[pick[1]].reshape(tokens, -1)
    old = rng.integers(0, 256, (2, n_pages, heads, page, 64), dtype=np.uint8)
    want = old.copy()
    for which, (meta, part) in enumerate(((meta_k, rows[:, :heads * 128]), (meta_v, rows[:, -heads * 128:]))):
        there = (slots >= 0) & (slots < n_pages * page)
        if there.any():
            blocks, _ = eo.encode(meta, np.ascontiguousarray(part[there]), eo.SELECT_MINMAX)
            want[which, slots[there] // page, :, slots[there] % page] = blocks.reshape(-1, heads, 64)
    d_rows, d_pools = torch.from_numpy(rows).cuda(), torch.from_numpy(old).cuda()
    d_meta = [B.meta_to_device(lib_meta_from_oracle(B, m)) for m in (meta_k, meta_v)]
    cache = B.paged_cache(d_meta[0], d_meta[1], d_pools[0], d_pools[1], n_pages, heads, page)
    at = d_rows.data_ptr()
    B.ecco_paged_append(cache, at, at + 2 * (heads * 128 + extra), rows.shape[1], ints(slots), tokens)
    assert np.array_equal(d_pools.cpu().numpy(), want)
    assert B.ecco_device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,heads", [(1023, 8), (1024, 8), (2731, 3), (8191, 8), (8192, 8), (10239, 8), (10240, 8), (27307, 3), (1300, 64)])
def test_append_gives_the_blocks_of_kv_compress(B, dev, eo, kv_small, tokens, heads):
    """On both sides of the lines between the two compressors and between one launch and two, with metadata of their own for K and V."""
    rng = np.random.default_rng([70, tokens])
    meta_v = eo.calibrate(kv_small["cal"].reshape(-1)[:128 * 512], S=16, H=4, seed=9, select=eo.SELECT_MINMAX)
    d_meta = [B.meta_to_device(lib_meta_from_oracle(B, m)) for m in (kv_small["meta"], meta_v)]
    src = torch.from_numpy(kv_small["k"].reshape(-1, 128)).cuda()
    x = src[torch.from_numpy(rng.integers(0, len(src), (tokens, 2, heads))).cuda()]
    page = 16
    pages = tokens // page + 2
    slots = torch.from_numpy(rng.permutation(pages * page)[:tokens]).cuda()
    pools = [torch.zeros((pages, heads, page, 64), dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = B.paged_cache(*d_meta, *pools, pages, heads, page)
    B.ecco_paged_append(cache, x.data_ptr(), x.data_ptr() + heads * 256, 2 * heads * 128, slots.int(), tokens)
    for which in range(2):
        rows = x[:, which].contiguous()
        want = torch.empty((tokens, heads, 64), dtype=torch.uint8, device="cuda")
        B.ecco_kv_compress(d_meta[which], rows, tokens * heads, want)
        assert torch.equal(pools[which].permute(0, 2, 1, 3).reshape(pages * page, heads, 64)[slots], want), which
    assert B.ecco_device_status() == 0


# ------------------------------------------------------------------ attention
class Paged:
    """Requests of given lengths over pools of blocks drawn from the oracle-encoded cache."""

    def __init__(self, B, eo, metas, blocks, new, kv, heads, g, page, seed=0, q_extra=0):
        rng = np.random.default_rng([seed, heads, g, page])
        self.B, self.heads, self.g, self.page, self.new, self.kv = B, heads, g, page, list(new), list(kv)
        n_req, held = len(new), [-(-k // page) for k in kv]
        self.n_pages = sum(held) + 3
        self.pools = [b[rng.integers(0, len(b), (self.n_pages, heads, page))] for b in blocks]
        self.stride = max(held + [0]) + 2
        self.tables = rng.integers(-3, 1 << 30, (n_req, self.stride)).astype(np.int32)           # arbitrary behind a request's pages
        ids, at = rng.permutation(self.n_pages), 0
        for r, h in enumerate(held):
            self.tables[r, :h] = ids[at:at + h]
            at += h
        self.tokens = sum(new)
        self.q_stride = heads * g * 128 + q_extra
        self.q = rng.standard_normal((self.tokens, self.q_stride)).astype(np.float16)
        self.decoded = []                                                     # per request [kv][heads][128], fp64
        for pool, meta in zip(self.pools, metas):
            self.decoded.append([])
            for r, k in enumerate(kv):
                t = np.arange(k)
                b = pool[self.tables[r, t // page], :, t % page].reshape(-1, 64)
                with np.errstate(over="ignore"):
                    x = eo.decode(meta, b).astype(np.float64) if k else np.zeros((0, 128))
                self.decoded[-1].append(np.clip(x, -65504, 65504).reshape(k, heads, 128))
        self.d_meta = [B.meta_to_device(lib_meta_from_oracle(B, m)) for m in metas]
        self.d_pools = [torch.from_numpy(p).cuda() for p in self.pools]
        self.cache = B.paged_cache(self.d_meta[0], self.d_meta[1], self.d_pools[0], self.d_pools[1], self.n_pages, heads, page)
        self.d_tables, self.d_q = ints(self.tables), torch.from_numpy(self.q).cuda()
        tiles = np.concatenate([[0], np.cumsum([-(-k // 32) for k in kv])])
        self.d_cu, self.d_lens, self.d_tiles = ints(np.concatenate([[0], np.cumsum(new)])), ints(kv), ints(tiles)
        self.batch = B.paged_batch(self.d_tables, self.stride, self.d_cu, self.d_lens, self.d_tiles, n_req, self.tokens, max(new), max(kv), int(tiles[-1]))

    def run(self, causal, scale=128 ** -0.5, ws_bytes=None, lse=True, spare=2, batch=None):
        B, own = self.B, self.batch
        self.batch = batch or own
        full = B.ecco_paged_attn_workspace_bytes(self.cache, self.batch, self.g)
        ws_bytes = full if ws_bytes is None else ws_bytes
        ws = torch.full((ws_bytes,), 0xff, dtype=torch.uint8, device="cuda")  # NaN, whatever it is read as
        out = torch.full((self.tokens + spare, self.heads * self.g, 128), 7.0, dtype=torch.float16, device="cuda")
        d_lse = torch.full((self.tokens + spare, self.heads * self.g), 7.0, device="cuda") if lse else None
        B.ecco_paged_attn(self.cache, self.batch, self.g, self.d_q, self.q_stride, scale, B.ATTN_CAUSAL if causal else 0, out, d_lse, ws, ws_bytes)
        torch.cuda.synchronize()
        self.batch = own
        assert (out[self.tokens:] == 7).all()                                  # rows behind the last request
        return out[:self.tokens].cpu().numpy(), d_lse[:self.tokens].cpu().numpy() if lse else None

    def check(self, out, lse, causal, scale=128 ** -0.5, rows=None):
        at = 0
        for r, (n, kv) in enumerate(zip(self.new, self.kv)):
            k, v = self.decoded[0][r], self.decoded[1][r]
            picked = range(n) if rows is None else [i for i in range(n) if (at + i) % rows == 0 or i == n - 1]
            for i in picked:
                see = min(max(kv - n + i + 1, 0), kv) if causal else kv
                for hq in range(self.heads * self.g):
                    got, got_lse = out[at + i, hq].astype(np.float64), None if lse is None else float(lse[at + i, hq])
                    if see == 0:
                        assert not got.any() and (lse is None or got_lse == -math.inf), (r, i, hq)
                        continue
                    q, kk, vv = self.q[at + i, hq * 128:(hq + 1) * 128].astype(np.float64), k[:see, hq // self.g], v[:see, hq // self.g]
                    s = scale * (kk @ q)
                    top = s.max()
                    p = np.exp(s - top)
                    ref, mass, ref_lse = p @ vv / p.sum(), p @ np.abs(vv) / p.sum(), top + math.log(p.sum())
                    e_s = 128 * 2.0 ** -23 * abs(scale) * (np.abs(kk) @ np.abs(q)).max() + 2.0 ** -22 * (1 + np.abs(s).max())
                    sums = (see / 16 + 32) * 2.0 ** -23
                    tol = 2.0 ** -11 * np.abs(ref) + (2.0 ** -11 + 2 * e_s + sums) * mass + 2.0 ** -32 * np.abs(vv).sum(0) + 2.0 ** -25
                    assert (np.abs(got - ref) <= tol).all(), (r, i, hq, float((np.abs(got - ref) / tol).max()))
                    if lse is not None:
                        assert abs(got_lse - ref_lse) <= e_s + sums + 2.0 ** -22 * abs(ref_lse) + 2.0 ** -20, (r, i, hq, got_lse, ref_lse)
            at += n


@pytest.fixture(scope="session")
def caches(eo, kv_small, synth):
    """(metadata, blocks) of a K and of a V cache with tables of their own."""
    v = synth.kv_cache(2, 2, 256, 1004, 3004)
    meta_v = eo.calibrate(synth.kv_cache(2, 2, 256, 2004, 3004), S=64, H=4, seed=4, select=eo.SELECT_MINMAX)
    blocks_v, _ = eo.encode(meta_v, v, eo.SELECT_MINMAX)
    return (kv_small["meta"], meta_v), (kv_small["blocks"].reshape(-1, 64), blocks_v.reshape(-1, 64))


SHAPES = [
    # new tokens, cached tokens (new ones among them where causal), KV heads, query heads per KV head, page size
    ([1], [1], 1, 1, 1),
    ([1], [33], 2, 4, 16),
    ([1, 1, 1], [777, 1, 64], 8, 4, 16),
    ([1] * 40, [1 + 37 * i % 700 for i in range(40)], 2, 8, 32),
    ([1, 0, 1, 1], [31, 50, 0, 32], 3, 16, 8),                                # no new token; no token at all
    ([5, 3, 8], [100, 3, 4000], 2, 2, 64),
    ([4, 1, 2], [129, 2, 1000], 2, 5, 128),
    ([7, 2], [3, 300], 1, 4, 4),                                               # more new tokens than the cache holds: rows that see nothing
    ([33, 1], [40, 2000], 2, 3, 16),
    ([64, 17], [64, 500], 1, 16, 4096),
    ([130, 1, 257], [700, 900, 257], 2, 4, 16),
    ([100], [3000], 1, 1, 2),
    ([61, 40], [200, 129], 1, 7, 32),                                          # heads that do not divide 128: blocks of whole tokens
    ([50], [333], 2, 13, 16),
    ([20, 1, 18], [0, 0, 5], 1, 2, 16),                                        # many rows and no token at all; one tile
    ([128, 129], [128, 1025], 1, 2, 64),                                       # a block that is just full, and one row more
]


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("shape", SHAPES, ids=[str(i) for i in range(len(SHAPES))])
def test_attention_matches_64_bits(B, dev, eo, caches, shape, causal):
    new, kv, heads, g, page = shape
    p = Paged(B, eo, *caches, new, kv, heads, g, page, seed=len(new), q_extra=64 if g == 4 else 0)
    out, lse = p.run(causal)
    p.check(out, lse, causal)
    assert B.ecco_device_status() == 0
    again, _ = p.run(causal, lse=False)
    assert np.array_equal(out.view(np.uint16), again.view(np.uint16))          # reproducible, with and without lse


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [0.0, -0.11, 1.0, 1e-42])
def test_attention_scales(B, dev, eo, caches, scale):
    """Zero (all tokens alike), negative, sharp, below fp32's normal range; few rows and many."""
    p = Paged(B, eo, *caches, [1, 40, 3], [100, 300, 2], 2, 2, 16, seed=7)
    for causal in (True, False):
        out, lse = p.run(causal, scale=scale)
        p.check(out, lse, causal, scale=float(np.float32(scale)))


@pytest.mark.gpu
def test_attention_takes_some_heads_at_a_time(B, dev, eo, caches):
    p = Paged(B, eo, *caches, [1, 70, 4], [500, 90, 64], 5, 3, 16, seed=8)
    sizes = []
    for heads in (1, 2, 3, 5):
        c = B.paged_cache(p.d_meta[0], p.d_meta[1], p.d_pools[0], p.d_pools[1], p.n_pages, heads, p.page)
        sizes.append(B.ecco_paged_attn_workspace_bytes(c, p.batch, p.g))
    assert sizes == sorted(sizes) and sizes[0] < sizes[-1]
    for n in sizes:
        out, lse = p.run(True, ws_bytes=n)
        p.check(out, lse, True, rows=3)

    def launches(n):
        before = B.ecco_kernel_launch_count()
        out, lse = p.run(True, ws_bytes=n)
        p.check(out, lse, True, rows=7)
        return B.ecco_kernel_launch_count() - before

    low, high = 0, sizes[0]                                                    # what one head needs on this device: at most what the call says
    while high - low > 16:
        mid = (low + high) // 2
        try:
            p.run(True, ws_bytes=mid)
            high = mid
        except B.EccoError as e:
            assert e.code == B.ERR_WORKSPACE
            low = mid
    assert low > 2 * 20 * 8192 and launches(high) == 5 * launches(sizes[-1])
    with pytest.raises(B.EccoError) as ei:
        B.ecco_paged_attn(p.cache, p.batch, p.g, p.d_q, p.q_stride, 0.1, 0, p.d_q, None, None, 1 << 40)
    assert ei.value.code == B.ERR_WORKSPACE


@pytest.mark.gpu
def test_attention_of_a_padded_batch(B, dev, eo, caches):
    """Sizes that the host passes are upper bounds: spare rows, requests without tokens at the end, generous maxima; an odd workspace address."""
    p = Paged(B, eo, *caches, [1, 30, 0, 0], [70, 64, 0, 0], 2, 4, 16, seed=9)
    for new, kv, tiles in ((30, 70, 5), (900, 5000, 300), (31, 71, 6)):
        b = B.paged_batch(p.d_tables, p.stride, p.d_cu, p.d_lens, p.d_tiles, 4, p.tokens + 2, new, kv, tiles)
        q = torch.cat([p.d_q, torch.full((2, p.q_stride), math.nan, dtype=torch.float16, device="cuda")])
        ws = torch.full((B.ecco_paged_attn_workspace_bytes(p.cache, b, p.g) + 16,), 0xff, dtype=torch.uint8, device="cuda")[16:]
        out = torch.full((p.tokens + 2, 8, 128), 7.0, dtype=torch.float16, device="cuda")
        lse = torch.full((p.tokens + 2, 8), 7.0, device="cuda")
        B.ecco_paged_attn(p.cache, b, p.g, q, p.q_stride, 0.1, B.ATTN_CAUSAL, out, lse, ws, ws.numel())
        assert (out[p.tokens:] == 7).all() and (lse[p.tokens:] == 7).all()
        p.check(out[:p.tokens].cpu().numpy(), lse[:p.tokens].cpu().numpy(), True, scale=0.1)
    assert B.ecco_device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("new,kv,heads,g", [([1, 1, 1], [300, 1, 64], 3, 1), ([1, 0, 1, 1], [2000, 5, 0, 33], 2, 1), ([1, 1], [70, 129], 2, 2), ([2, 1, 2], [90, 1, 2], 1, 1),
                                            ([1] * 260, list(range(260)), 1, 2), ([2, 1], [40, 64], 2, 4), ([20, 1], [100, 300], 1, 3),
                                            ([1, 0, 1], [700, 3, 31], 2, 3), ([2, 1, 0, 2], [33, 500, 0, 2], 3, 3), ([3, 1], [3, 77], 1, 2), ([5, 7], [64, 7], 1, 1),
                                            ([1] * 260, list(range(260)), 1, 8), ([3, 1], [90, 300], 2, 3)])
def test_attention_of_large_calls(B, dev, eo, caches, new, kv, heads, g, causal):
    """The ways of a call whose bounds say that it is large: K and V in every CTA, and, for up to eight rows to a request, products with K
    instead of K in tiles."""
    p = Paged(B, eo, *caches, new, kv, heads, g, 16, seed=41)
    b = B.paged_batch(p.d_tables, p.stride, p.d_cu, p.d_lens, p.d_tiles, len(new), p.tokens, max(new), max(kv), 28000 // heads + 1)
    out, lse = p.run(causal, batch=b)
    p.check(out, lse, causal)
    small, _ = p.run(causal)
    assert B.ecco_device_status() == 0
    top = max(np.abs(v).max() for v in p.decoded[1] if len(v))
    assert (np.abs(out.astype(np.float64) - small) <= 2.0 ** -10 * np.abs(small) + 2.0 ** -10 * top).all()


@pytest.mark.gpu
def test_attention_of_more_requests_than_shared_memory_keeps(B, dev, eo, caches):
    rng = np.random.default_rng(10)
    new = rng.integers(0, 4, 300)
    new[[5, 77, 299]] = [40, 9, 130]
    kv = new + rng.integers(0, 60, 300)
    p = Paged(B, eo, *caches, new.tolist(), kv.tolist(), 1, 2, 8, seed=10)
    out, lse = p.run(True)
    p.check(out, lse, True)


@pytest.mark.gpu
@pytest.mark.parametrize("new", [[1, 2], [40, 30]])
def test_values_beyond_fp16_do_not_leave_their_rows(B, dev, eo, caches, new):
    """V values beyond fp16's range enter as +-65504; a row that does not see them has nothing of them."""
    metas, blocks = caches
    big = eo.Meta()
    ctypes.memmove(ctypes.byref(big), ctypes.byref(metas[1]), ctypes.sizeof(big))
    big.e = 16
    p = Paged(B, eo, (metas[0], big), blocks, new, [50, 40], 2, 2, 16, seed=11)
    assert (np.abs(p.decoded[1][0]) == 65504).any()
    out, lse = p.run(True)
    p.check(out, lse, True)
    # K beyond fp16's range, in tiles and taken at once: scores are what finite numbers give
    k = Paged(B, eo, (big, metas[1]), (blocks[1], blocks[1]), [1, 2], [50, 40], 2, 1, 16, seed=15)
    assert (np.abs(k.decoded[0][0]) == 65504).any()
    for bound, tiles in ((2, 4), (2, 7000), (3, 14000)):
        got, got_lse = k.run(True, scale=1e-6, batch=B.paged_batch(k.d_tables, k.stride, k.d_cu, k.d_lens, k.d_tiles, 2, k.tokens, bound, 50, tiles))
        k.check(got, got_lse, True, scale=float(np.float32(1e-6)))
    # and a q that is not finite stays in the rows of its token
    clean = out.copy()
    p.d_q[0, :256] = math.inf
    out, _ = p.run(True)
    assert np.array_equal(out[1:].view(np.uint16), clean[1:].view(np.uint16)) and np.array_equal(out[0, 2:].view(np.uint16), clean[0, 2:].view(np.uint16))


@pytest.mark.gpu
@pytest.mark.parametrize("new,g,tiles", [([1, 2], 2, 0), ([1, 2], 1, 14000), ([1, 2], 2, 14000), ([1, 2], 4, 7000), ([40, 30], 2, 0), ([150, 3], 2, 0)])
def test_a_q_that_is_no_number_gives_none(B, dev, eo, caches, new, g, tiles):
    """In requests that one run of tiles holds and in cut ones; the other tokens' rows stay as they are."""
    for kv in ([150, 200], [5000, 3000]):
        p = Paged(B, eo, *caches, new, kv, 2, g, 16, seed=19)
        bound = B.paged_batch(p.d_tables, p.stride, p.d_cu, p.d_lens, p.d_tiles, 2, p.tokens, max(new), max(kv), tiles) if tiles else None
        want, want_lse = p.run(True, batch=bound)
        p.d_q[new[0], 5] = math.nan                        # the first query head of the second request's first token
        out, lse = p.run(True, batch=bound)
        assert np.isnan(out[new[0], 0]).all() and np.isnan(lse[new[0], 0])
        rest = np.ones(out.shape[:2], bool)
        rest[new[0], 0] = False
        assert np.array_equal(out[rest].view(np.uint16), want[rest].view(np.uint16)) and np.array_equal(lse[rest], want_lse[rest])
    assert B.ecco_device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("new", [[1, 2, 1], [30, 33, 60]])
def test_bad_pages_and_lengths_are_reported(B, dev, eo, caches, new):
    """The requests beside a broken one keep their results, and nothing outside of the buffers is touched."""
    def make():
        return Paged(B, eo, *caches, new, [100, 90, 200], 2, 2, 16, seed=12)

    p = make()
    for page in (-1, p.n_pages, 2**31 - 1, -2**31):
        p.d_tables[1, 2] = page
        out, lse = p.run(True)
        assert B.ecco_device_status() == B.ERR_INVALID_ARG
        q = make()
        q.new, q.kv = p.new, p.kv
        keep = np.r_[0:new[0], new[0] + new[1]:sum(new)]
        want, want_lse = q.run(True)
        assert np.array_equal(out[keep].view(np.uint16), want[keep].view(np.uint16)) and np.array_equal(lse[keep], want_lse[keep])
    # lengths and prefix sums that say more than the bounds, or anything at all
    rng = np.random.default_rng(13)
    for name in ("d_lens", "d_tiles", "d_cu", "d_tables"):
        for trial in range(6):
            p = make()
            t = getattr(p, name)
            t.copy_(torch.from_numpy(rng.integers(-2**31, 2**31, t.shape) if trial < 3 else rng.integers(-50, 300, t.shape)).int())
            p.run(True, spare=0)
            assert B.ecco_device_status() in (0, B.ERR_INVALID_ARG)
    p = make()
    out, lse = p.run(True)
    p.check(out, lse, True, rows=5)
    assert B.ecco_device_status() == 0


@pytest.mark.gpu
def test_pools_beyond_32_bits(B, dev, eo, caches):
    """Pages on both sides of byte 2^32 of a pool; append and attention."""
    heads, page = 32, 64
    n_pages = (1 << 32) // (heads * page * 64) + 40
    pool = torch.empty((n_pages, heads, page, 64), dtype=torch.uint8, device="cuda")
    (meta, _), _ = caches
    d_meta = B.meta_to_device(lib_meta_from_oracle(B, meta))
    cache = B.paged_cache(d_meta, d_meta, pool, pool, n_pages, heads, page)
    ids = [n_pages - 1, 3, n_pages - 39, n_pages - 41]
    kv = 3 * page + 5
    slots = np.concatenate([np.arange(e * page, e * page + page) for e in ids])[:kv]
    rng = np.random.default_rng(14)
    x = rng.standard_normal((kv, heads * 128)).astype(np.float16)
    B.ecco_paged_append(cache, torch.from_numpy(x).cuda(), torch.from_numpy(x).cuda(), heads * 128, ints(slots), kv)
    blocks, _ = eo.encode(meta, x, eo.SELECT_MINMAX)
    got = pool[torch.from_numpy(slots // page).cuda(), :, torch.from_numpy(slots % page).cuda()].cpu().numpy()
    assert np.array_equal(got.reshape(-1, 64), blocks)
    values = eo.decode(meta, blocks).astype(np.float64).reshape(kv, heads, 128)
    q = rng.standard_normal((2, heads * 128)).astype(np.float16)
    batch = B.paged_batch(ints([ids]), 4, ints([0, 2]), ints([kv]), ints([0, -(-kv // 32)]), 1, 2, 2, kv, -(-kv // 32))
    n = B.ecco_paged_attn_workspace_bytes(cache, batch, 1)
    out = torch.empty((2, heads, 128), dtype=torch.float16, device="cuda")
    B.ecco_paged_attn(cache, batch, 1, torch.from_numpy(q).cuda(), heads * 128, 0.1, 0, out, None, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    for h in range(heads):
        s = 0.1 * (q[:, h * 128:(h + 1) * 128].astype(np.float64) @ values[:, h].T)
        w = np.exp(s - s.max(1, keepdims=True))
        w /= w.sum(1, keepdims=True)
        ref, mass = w @ values[:, h], w @ np.abs(values[:, h])
        assert (np.abs(out[:, h].cpu().numpy() - ref) <= 2.0 ** -11 * np.abs(ref) + (2.0 ** -11 + 2.0 ** -14) * mass + 2.0 ** -25).all(), h


# ------------------------------------------------------------------ the three together
class Server:
    """Requests that grow: every step plans, appends and attends, on fixed buffers."""

    def __init__(self, B, eo, caches, n_req, heads, g, page, max_kv, seed):
        (self.metas, _), self.B, self.eo = caches, B, eo
        self.heads, self.g, self.page, self.rng = heads, g, page, np.random.default_rng(seed)
        self.stride = max_kv // page + 1
        self.n_pages = n_req * self.stride
        self.max_new, self.max_kv = 48, max_kv
        self.n_tokens = n_req * self.max_new
        z = lambda *shape, dtype=torch.int32: torch.zeros(shape, dtype=dtype, device="cuda")  # noqa: E731
        self.ctx, self.new, self.tables = z(n_req), z(n_req), z(n_req, self.stride)
        self.free = torch.from_numpy(self.rng.permutation(self.n_pages)).int().cuda()
        self.used = 0
        self.slots, self.cu, self.lens, self.tiles, self.result = z(self.n_tokens), z(n_req + 1), z(n_req), z(n_req + 1), z(4)
        self.qkv = z(self.n_tokens, heads * (g + 2), 128, dtype=torch.float16)
        self.pools = [z(self.n_pages, heads, page, 64, dtype=torch.uint8) for _ in range(2)]
        self.d_meta = [B.meta_to_device(lib_meta_from_oracle(B, m)) for m in self.metas]
        self.cache = B.paged_cache(self.d_meta[0], self.d_meta[1], self.pools[0], self.pools[1], self.n_pages, heads, page)
        self.batch = B.paged_batch(self.tables, self.stride, self.cu, self.lens, self.tiles, n_req, self.n_tokens, self.max_new, max_kv, n_req * (max_kv // 32 + 1))
        self.ws_bytes = B.ecco_paged_attn_workspace_bytes(self.cache, self.batch, g)
        self.ws = z(self.ws_bytes, dtype=torch.uint8)
        self.out, self.lse = z(self.n_tokens, heads * g, 128, dtype=torch.float16), z(self.n_tokens, heads * g, dtype=torch.float32)
        self.free_now = self.free.clone()
        self.rows = [[] for _ in range(n_req)]                                # K and V values of every request so far

    def feed(self, new):
        """The host's part of a step: lengths and rows of the projection."""
        x = self.rng.standard_normal((self.n_tokens, self.heads * (self.g + 2), 128)).astype(np.float16)
        self.new.copy_(ints(new))
        self.qkv.copy_(torch.from_numpy(x))
        self.free_now[:self.n_pages - self.used] = self.free[self.used:]
        at = 0
        for r, n in enumerate(new):
            self.rows[r].append(x[at:at + n, self.heads * self.g:])
            at += n
        self.x = x

    def step(self):
        B, row = self.B, self.qkv.data_ptr()
        stride = self.heads * (self.g + 2) * 128
        B.ecco_paged_plan(self.page, self.n_pages, len(self.ctx), self.ctx, self.new, self.free_now, self.n_pages, self.tables, self.stride, self.slots,
                          self.n_tokens, self.cu, self.lens, self.tiles, self.result)
        B.ecco_paged_append(self.cache, row + self.heads * self.g * 256, row + self.heads * (self.g + 1) * 256, stride, self.slots, self.n_tokens)
        B.ecco_paged_attn(self.cache, self.batch, self.g, self.qkv.data_ptr(), stride, 128 ** -0.5, B.ATTN_CAUSAL, self.out, self.lse, self.ws, self.ws_bytes)

    def done(self):
        torch.cuda.synchronize()
        assert self.B.ecco_device_status() == 0 and self.result[0].item() == 0
        self.used += self.result[1].item()
        self.ctx.copy_(self.lens)
        return self.out.cpu().numpy(), self.lse.cpu().numpy()

    def check(self, out, lse, new):
        """A request's rows against 64 bits over all that it was ever given."""
        at = 0
        for r, n in enumerate(new):
            kv = np.concatenate(self.rows[r])
            if n and r % 3 == 0:
                p = Paged.__new__(Paged)
                p.heads, p.g, p.new, p.kv = self.heads, self.g, [n], [len(kv)]
                p.q = self.x[at:at + n, :self.heads * self.g].reshape(n, -1)
                p.decoded = []
                for which in range(2):
                    part = np.ascontiguousarray(kv[:, which * self.heads:(which + 1) * self.heads])
                    blocks, _ = self.eo.encode(self.metas[which], part, self.eo.SELECT_MINMAX)
                    p.decoded.append([self.eo.decode(self.metas[which], blocks).astype(np.float64).reshape(-1, self.heads, 128)])
                p.check(out[at:at + n], lse[at:at + n], True, rows=4)
            at += n


def steps_of(n_req):
    return [[37 - r % 30 for r in range(n_req)], [1] * n_req, [(r * 7) % 5 for r in range(n_req)], [0] * n_req, [48 if r == 1 else 1 for r in range(n_req)]]


@pytest.mark.gpu
def test_a_server_step_by_step(B, dev, eo, caches):
    s = Server(B, eo, caches, 6, 2, 2, 16, 160, 21)
    for new in steps_of(6):
        s.feed(new)
        s.step()
        out, lse = s.done()
        s.check(out, lse, new)


@pytest.mark.gpu
def test_captured_steps_replay_with_other_lengths(B, dev, eo, caches):
    """One step captured into a graph and replayed with other lengths, against the same steps issued one by one; two servers' graphs,
    each with a workspace of its own, on two streams at once."""
    eager = [Server(B, eo, caches, 6, 2, 2, 16, 160, seed) for seed in (22, 23)]
    graphed = [Server(B, eo, caches, 6, 2, 2, 16, 160, seed) for seed in (22, 23)]
    want = []
    for s in eager:
        want.append([])
        for new in steps_of(6):
            s.feed(new)
            s.step()
            want[-1].append(s.done())
    streams, graphs = [torch.cuda.Stream() for _ in graphed], []
    for s, stream in zip(graphed, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            s.step()
        graphs.append(g)
    for i, new in enumerate(steps_of(6)):
        for s in graphed:
            s.feed(new)
        torch.cuda.synchronize()
        for g, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                g.replay()
        for k, s in enumerate(graphed):
            out, lse = s.done()
            n = sum(new)
            assert np.array_equal(out[:n].view(np.uint16), want[k][i][0][:n].view(np.uint16)), (i, k)
            assert np.array_equal(lse[:n], want[k][i][1][:n]), (i, k)


@pytest.mark.gpu
def test_paged_and_dense_caches_agree(B, dev, eo, caches):
    """One token each over equal lengths: ecco_attn_scores and ecco_attn_values over the same blocks in one piece."""
    heads, g, kv, batch = 2, 4, 333, 3
    p = Paged(B, eo, *caches, [1] * batch, [kv] * batch, heads, g, 16, seed=31)
    out, _ = p.run(True)
    dense = [torch.from_numpy(np.stack([np.stack([pool[p.tables[r, np.arange(kv) // 16], h, np.arange(kv) % 16] for h in range(heads)]) for r in range(batch)])).cuda()
             for pool in p.pools]
    scores = torch.empty((batch, heads * g, kv), device="cuda")
    B.ecco_attn_scores(p.d_meta[0], dense[0], batch, heads, kv, g, p.d_q.view(batch, -1)[:, :heads * g * 128].contiguous(), 128 ** -0.5, scores)
    n = B.ecco_attn_values_workspace_bytes(batch, heads, kv, g)
    want = torch.empty((batch, heads * g, 128), device="cuda")
    B.ecco_attn_values(p.d_meta[1], dense[1], batch, heads, kv, g, scores, want, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    want = want.cpu().numpy().astype(np.float64)
    # both rounded: the tolerance of the paged call, with the largest |V| for the weighted mean
    top = max(np.abs(v).max() for v in p.decoded[1])
    assert (np.abs(out - want) <= 2.0 ** -11 * np.abs(want) + 2.0 ** -10 * top).all()


# ------------------------------------------------------------------ arrays that say more than the bounds
@pytest.mark.gpu
@pytest.mark.parametrize("new", [[2, 1, 3], [40, 33, 70]])
@pytest.mark.parametrize("what", ["more tokens than rows", "a request beyond the rows", "falling rows", "negative rows", "falling tiles", "negative tiles"])
def test_whatever_the_bounds_cut_off_is_reported(B, dev, eo, caches, new, what):
    """Rows of a request that were cut off would move the causal mask of those that are left: the status says so, the requests in front keep
    their results, and the rows behind the bound stay as they are."""
    p = Paged(B, eo, *caches, new, [100, 90, 200], 2, 2, 16, seed=51)
    want, want_lse = p.run(True)
    assert B.ecco_device_status() == 0
    n = p.tokens
    if what == "more tokens than rows":
        n -= 1
    elif what == "a request beyond the rows":
        n -= new[2]
    elif what == "falling rows":
        p.d_cu[2] = new[0] - 1
    elif what == "negative rows":
        p.d_cu[0] = -1
    elif what == "falling tiles":                                              # of a request without a token, so its own length still fits
        p.d_lens[1] = 0
        p.d_tiles[2] = 3
    else:
        p.d_tiles[0] = -1
    b = B.paged_batch(p.d_tables, p.stride, p.d_cu, p.d_lens, p.d_tiles, 3, n, max(new) + 2, 200, p.batch.max_tiles)
    out, lse = p.run(True, batch=b)
    assert B.ecco_device_status() == B.ERR_INVALID_ARG
    if "negative" not in what:
        assert np.array_equal(out[:new[0] - 1].view(np.uint16), want[:new[0] - 1].view(np.uint16)) and np.array_equal(lse[:new[0] - 1], want_lse[:new[0] - 1])
    assert (out[n:] == 7).all() and (lse[n:] == 7).all()
    assert B.ecco_device_status() == 0                                         # told once


@pytest.mark.gpu
@pytest.mark.parametrize("g", [1, 16])
def test_prefix_sums_whose_lengths_pass_32_bits(B, dev, eo, caches, g):
    """65535 requests that all say that they have 70000 tiles or none, 2.3e9 in all: the line of tiles ends at the 70000 that there are.
    Everything that the call may write lies between guards."""
    (meta, _), (blocks, _) = caches
    n, tiles = 65535, 70000
    d_meta = B.meta_to_device(lib_meta_from_oracle(B, meta))
    pool = torch.from_numpy(blocks[:64].reshape(1, 1, 64, 64).copy()).cuda()
    cache = B.paged_cache(d_meta, d_meta, pool, pool, 1, 1, 64)
    sums = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    sums[1::2] = tiles
    assert int(sums.diff().clamp(min=0).sum(dtype=torch.int64)) > 2**31
    batch = B.paged_batch(torch.zeros((n, 1), dtype=torch.int32, device="cuda"), 1, torch.arange(n + 1, dtype=torch.int32, device="cuda"),
                          torch.full((n,), 64, dtype=torch.int32, device="cuda"), sums, n, n, 1, 64, tiles)
    need = B.ecco_paged_attn_workspace_bytes(cache, batch, g)
    ws = torch.full((need + 8192,), 0xa5, dtype=torch.uint8, device="cuda")
    out = torch.full((n + 16, g, 128), 7.0, dtype=torch.float16, device="cuda")
    lse = torch.full((n + 16, g), 7.0, device="cuda")
    q = torch.randn((n, g, 128), device="cuda").half()
    B.ecco_paged_attn(cache, batch, g, q, g * 128, 0.1, 0, out[8:], lse[8:], ws[4096:], need)
    assert B.ecco_device_status() == B.ERR_INVALID_ARG
    assert (ws[:4096] == 0xa5).all() and (ws[4096 + need:] == 0xa5).all()
    assert all((t[:8] == 7).all() and (t[n + 8:] == 7).all() for t in (out, lse))
    assert np.array_equal(pool.cpu().numpy().reshape(-1, 64), blocks[:64])
    p = Paged(B, eo, *caches, [1, 3], [300, 70], 2, 2, 16, seed=52)             # and the next call is as ever
    got, got_lse = p.run(True)
    p.check(got, got_lse, True)
    assert B.ecco_device_status() == 0


# ------------------------------------------------------------------ calls behind one another
class Layers:
    """Layers of one step: append and attention of each, its rows the output of the one before; one workspace for all."""

    def __init__(self, B, eo, caches, n, new, kv, heads, g, page, tiles=0, small=False, seed=60):
        self.B, self.g, self.row = B, g, heads * g * 128
        self.p = [Paged(B, eo, *caches, new, kv, heads, g, page, seed=seed + i) for i in range(n)]
        p = self.p[0]
        self.heads = heads
        self.slots = [ints([q.tables[r, t // page] * page + t % page for r in range(len(new)) for t in range(kv[r] - new[r], kv[r])]) for q in self.p]
        assert g >= 2                                                          # K and V of a layer are parts of its rows
        self.first = torch.from_numpy(p.q[:, :self.row].copy()).cuda()
        self.batch = [B.paged_batch(q.d_tables, q.stride, q.d_cu, q.d_lens, q.d_tiles, len(new), q.tokens, max(new), max(kv), tiles or q.batch.max_tiles) for q in self.p]
        one = B.paged_cache(p.d_meta[0], p.d_meta[1], p.d_pools[0], p.d_pools[1], p.n_pages, 1, page)
        self.ws_bytes = B.ecco_paged_attn_workspace_bytes(one if small else p.cache, self.batch[0], g)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device="cuda")
        self.outs = [torch.empty((p.tokens, heads * g, 128), dtype=torch.float16, device="cuda") for _ in range(n)]

    def reset(self):
        for q in self.p:
            for d, h in zip(q.d_pools, q.pools):
                d.copy_(torch.from_numpy(h))
        for o in self.outs:
            o.fill_(math.nan)
        self.ws.fill_(0xff)

    def step(self, after=lambda: None):
        x = self.first
        for q, batch, slots, out in zip(self.p, self.batch, self.slots, self.outs):
            self.B.ecco_paged_append(q.cache, x.data_ptr(), x.data_ptr() + self.heads * 256, self.row, slots, q.tokens)
            after()
            self.B.ecco_paged_attn(q.cache, batch, self.g, x, self.row, 0.3, self.B.ATTN_CAUSAL, out, None, self.ws, self.ws_bytes)
            after()
            x = out

    def results(self):
        return [t.cpu().numpy().view(np.uint8) for t in self.outs + [d for q in self.p for d in q.d_pools]]


LAYERS = {
    "few rows": dict(new=[1, 2, 1, 3], kv=[700, 90, 3000, 3], heads=3, g=3, page=16),
    "many rows": dict(new=[40, 130, 257], kv=[700, 130, 900], heads=2, g=2, page=32),
    "both": dict(new=[1, 40, 3, 130, 1, 2], kv=[2700, 300, 50, 500, 64, 900], heads=2, g=4, page=16),
    "both, some heads at a time": dict(new=[1, 40, 3, 130, 1, 2], kv=[2700, 300, 50, 500, 64, 900], heads=3, g=4, page=16, small=True),
    "large, two rows": dict(new=[1, 1, 1], kv=[900, 64, 3000], heads=2, g=2, page=16, tiles=14000),
    "large, six rows": dict(new=[2, 1, 1], kv=[900, 64, 3000], heads=2, g=3, page=16, tiles=14000),
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", LAYERS)
def test_layers_behind_one_another_on_one_workspace(B, dev, eo, caches, name):
    """Nothing waits on the host between the calls, every call reads what the one before wrote, and all use one workspace: as with a
    synchronisation behind every call."""
    s = Layers(B, eo, caches, 6, **LAYERS[name])
    s.reset()
    s.step(after=torch.cuda.synchronize)
    want = s.results()
    assert all(np.isfinite(o.view(np.float16)).all() for o in want[:6])
    for _ in range(5):
        s.reset()
        s.step()
        for i, (w, g) in enumerate(zip(want, s.results())):
            assert np.array_equal(w, g), i
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.step()
    for _ in range(3):
        s.reset()
        graph.replay()
        for i, (w, g) in enumerate(zip(want, s.results())):
            assert np.array_equal(w, g), i
    assert B.ecco_device_status() == 0


@pytest.mark.gpu
def test_callers_on_several_host_threads(B, dev, eo, caches):
    """Four threads, each with a stream, layers and a workspace of its own, at once."""
    import threading

    makers = ["few rows", "many rows", "both", "large, six rows"]
    all_layers, want = [], []
    for i, name in enumerate(makers):
        s = Layers(B, eo, caches, 3, **LAYERS[name], seed=80 + 10 * i)
        s.reset()
        s.step(after=torch.cuda.synchronize)
        want.append(s.results())
        all_layers.append(s)
    got, errors, gate = [None] * len(makers), [], threading.Barrier(len(makers))

    def work(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(10):
                    all_layers[i].reset()
                    stream.synchronize()
                    gate.wait(60)
                    for _ in range(3):                                         # the pools' new slots get the same blocks again
                        all_layers[i].step()
                    stream.synchronize()
                    got[i] = all_layers[i].results()
                    for w, g in zip(want[i], got[i]):
                        assert np.array_equal(w, g), makers[i]
        except BaseException as e:                                             # told by the main thread
            errors.append(e)
            gate.abort()

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(makers))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    assert B.ecco_device_status() == 0


# ------------------------------------------------------------------ nothing outside of the buffers
class Guarded:
    """A buffer between two stretches of a known pattern."""
    EDGE = 1 << 16

    def __init__(self, shape, dtype, fill=None):
        size = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
        self.all = torch.full((size + 2 * self.EDGE + 256,), 0xa5, dtype=torch.uint8, device="cuda")
        self.at = self.EDGE + -(self.all.data_ptr() + self.EDGE) % 256
        self.size = size
        self.body = self.all[self.at:self.at + size].view(dtype).view(shape)
        if fill is not None:
            self.body.copy_(fill) if isinstance(fill, torch.Tensor) else self.body.fill_(fill)

    def check(self, what):
        assert (self.all[:self.at] == 0xa5).all() and (self.all[self.at + self.size:] == 0xa5).all(), what


def arbitrary(rng, t, kind, largest):
    """Any numbers, numbers in range, the extremes, or numbers in range that only rise."""
    if kind == "any":
        a = rng.integers(-2**31, 2**31, t.shape)
    elif kind == "extremes":
        a = rng.choice([-2**31, 2**31 - 1, -1, 0, 1, largest, largest + 1], t.shape)
    else:
        a = rng.integers(-2, largest + 2, t.shape)
        if kind == "rising":
            a = np.sort(a, axis=None).reshape(t.shape)
    t.copy_(torch.from_numpy(a).int())


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["few rows", "many rows", "both", "both, one head at a time", "large, one row", "large, two rows", "large, eight rows", "large, many rows"])
def test_attention_of_arbitrary_arrays_stays_in_its_buffers(B, dev, eo, caches, form):
    new, g, heads, tiles = {"few rows": ([1, 2, 1, 4], 3, 2, 0), "many rows": ([40, 33, 270, 60], 2, 2, 0), "both": ([1, 40, 3, 130], 4, 2, 0),
                            "both, one head at a time": ([1, 40, 3, 130], 4, 3, 0), "large, one row": ([1] * 4, 1, 2, 14000), "large, two rows": ([1] * 4, 2, 2, 14000),
                            "large, eight rows": ([2, 1, 1, 2], 4, 2, 14000), "large, many rows": ([70, 40, 33, 1], 2, 2, 14000)}[form]
    p = Paged(B, eo, *caches, new, [100, 90, 700, 200], heads, g, 16, seed=53)
    n, clean_tiles = p.tokens, p.batch.max_tiles
    tiles = tiles or clean_tiles
    names = ("d_tables", "d_cu", "d_lens", "d_tiles")
    clean = {name: getattr(p, name).clone() for name in names}
    largest = {"d_tables": p.n_pages, "d_cu": n, "d_lens": 700, "d_tiles": tiles}
    batch = B.paged_batch(p.d_tables, p.stride, p.d_cu, p.d_lens, p.d_tiles, 4, n, max(new), 700, tiles)
    size = p.cache
    if "one head" in form:
        size = B.paged_cache(p.d_meta[0], p.d_meta[1], p.d_pools[0], p.d_pools[1], p.n_pages, 1, p.page)
    need = B.ecco_paged_attn_workspace_bytes(size, batch, g)
    ws, out, lse = Guarded((need,), torch.uint8, 0xff), Guarded((n, heads * g, 128), torch.float16, 7.0), Guarded((n, heads * g), torch.float32, 7.0)
    q0 = p.d_q.clone()
    run = lambda causal: B.ecco_paged_attn(p.cache, batch, g, p.d_q, p.q_stride, 0.1, causal, out.body, lse.body, ws.body, need)  # noqa: E731
    rng = np.random.default_rng([54, len(form)])
    for which in [(name,) for name in names] + [names[1:], names]:
        for kind in ("any", "extremes", "in range", "rising"):
            for name in names:
                getattr(p, name).copy_(clean[name])
            for name in which:
                arbitrary(rng, getattr(p, name), kind, largest[name])
            given = [getattr(p, name).clone() for name in names]
            run(int(rng.integers(2)))
            assert B.ecco_device_status() in (0, B.ERR_INVALID_ARG)
            for what, buffer in (("workspace", ws), ("out", out), ("lse", lse)):
                buffer.check((what, which, kind))
            assert torch.equal(p.d_q, q0) and all(torch.equal(getattr(p, name), was) for name, was in zip(names, given)), (which, kind)
            assert all(np.array_equal(d.cpu().numpy(), h) for d, h in zip(p.d_pools, p.pools)), (which, kind)
    for name in names:
        getattr(p, name).copy_(clean[name])
    run(1)
    assert B.ecco_device_status() == 0
    p.check(out.body.cpu().numpy(), lse.body.cpu().numpy(), True, scale=0.1, rows=5)


@pytest.mark.gpu
@pytest.mark.parametrize("n_req", [1, 5, 1500])
def test_plan_of_arbitrary_arrays_stays_in_its_buffers(B, dev, n_req):
    rng = np.random.default_rng([55, n_req])
    stride, n_slots, n_free, page, pages = 4, 3 * n_req + 2, n_req, 16, 2 * n_req + 1
    served = 0
    for kinds in [(a, b) for a in ("any", "extremes", "in range") for b in ("any", "extremes", "in range")] + [("fitting", "fitting")] * 3:
        t = {name: Guarded(shape, torch.int32, -7) for name, shape in dict(ctx=(n_req,), new=(n_req,), free=(n_free,), tables=(n_req, stride), slots=(n_slots,), cu=(n_req + 1,),
                                                                           lens=(n_req,), tiles=(n_req + 1,), result=(4,)).items()}
        if kinds[0] == "fitting":                          # lengths that can be served, over tables and free pages that say anything
            t["ctx"].body.copy_(ints(rng.integers(0, 15, n_req)))
            t["new"].body.copy_(ints(rng.integers(0, 4, n_req) * (np.arange(n_req) < 3 * n_req // 4)))
        else:
            arbitrary(rng, t["ctx"].body, kinds[0], 64)
            arbitrary(rng, t["new"].body, kinds[1], 3)
        for name in ("free", "tables"):
            arbitrary(rng, t[name].body, "extremes", pages)
        before = {name: b.body.clone() for name, b in t.items()}
        B.ecco_paged_plan(page, pages, n_req, t["ctx"].body, t["new"].body, t["free"].body, n_free, t["tables"].body, stride, t["slots"].body, n_slots, t["cu"].body,
                          t["lens"].body, t["tiles"].body, t["result"].body)
        for name, b in t.items():
            b.check((name, kinds))
        for name in ("ctx", "new", "free"):
            assert torch.equal(t[name].body, before[name]), (name, kinds)
        ctx, new = t["ctx"].body.cpu().numpy().astype(np.int64), t["new"].body.cpu().numpy().astype(np.int64)
        held, total = -(-ctx // page), -(-(ctx + new) // page)
        fine = (ctx >= 0).all() and (new >= 0).all() and (ctx + new <= page * stride).all()
        status = t["result"].body[0].item()
        assert status == (B.ERR_INVALID_ARG if not fine else B.ERR_WORKSPACE if new.sum() > n_slots or (total - held).sum() > n_free else 0), kinds
        if status:
            assert torch.equal(t["tables"].body, before["tables"]) and (t["slots"].body == -1).all() and not t["cu"].body.any() and not t["tiles"].body.any(), kinds
        else:
            want = plan_reference(page, pages, ctx, new, before["free"].cpu().numpy(), before["tables"].cpu().numpy(), n_slots)
            for name, w in zip(("tables", "slots", "cu", "lens", "tiles", "result"), want):
                assert np.array_equal(w, t[name].body.cpu().numpy()), (name, kinds)
            served += 1
    assert served >= 3


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,heads", [(7, 3), (600, 8), (2600, 8), (10500, 8)])
def test_append_to_arbitrary_slots_stays_in_the_pools(B, dev, eo, kv_small, tokens, heads):
    """Launches of either compressor, K and V in one and in two launches; places that no slot names stay as they are."""
    rng = np.random.default_rng([56, tokens])
    page, pages = 16, tokens // 8 + 2
    d_meta = B.meta_to_device(lib_meta_from_oracle(B, kv_small["meta"]))
    src = kv_small["k"].reshape(-1, 128)
    x = torch.from_numpy(src[rng.integers(0, len(src), tokens * 2 * heads)].reshape(tokens, -1)).cuda()
    for kind in ("any", "extremes", "in range"):
        pools = [Guarded((pages, heads, page, 64), torch.uint8, 0x3c) for _ in range(2)]
        cache = B.paged_cache(d_meta, d_meta, pools[0].body, pools[1].body, pages, heads, page)
        slots = torch.empty(tokens, dtype=torch.int32, device="cuda")
        arbitrary(rng, slots, kind, pages * page)
        B.ecco_paged_append(cache, x.data_ptr(), x.data_ptr() + heads * 256, 2 * heads * 128, slots, tokens)
        named = slots[(slots >= 0) & (slots < pages * page)].long()
        untouched = torch.ones(pages * page, dtype=torch.bool, device="cuda")
        untouched[named] = False
        for pool in pools:
            pool.check(kind)
            assert (pool.body.permute(0, 2, 1, 3).reshape(pages * page, -1)[untouched] == 0x3c).all(), kind
