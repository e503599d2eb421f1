"""The paged cache in 8 bits: ecco_paged8_append, ecco_paged8_attn.

Reference: the blocks in plain numpy, by their definition, bit for bit; attention in 64 bits over the values that the cache holds.
Tolerances of the attention, per output, from the kernels' roundings:
  scores: 128 products, exact in fp32, added on the tensor cores, which cut off: 128 * 2^-23 * scale * max_t sum |q k|; one rounding each of
          scale * log2(e), of its product with K's power of two (none, but where it leaves fp32), of the multiply-and-add and of the difference to
          the maximum, of numbers up to |s| + 15 + 7: 2^-22 * (|s| + 22);
  weights: fp16, half a step 2^-11 of each; exp2 2^-22; they stand at 2^7 times what they are relative to a reference that is at most the row's
          largest, so below fp16's normal range half a step is 2^-25 / 2^7 = 2^-32 of that: for many rows of the largest weight, for few of
          the largest weight times power of two, times an E4M3 number;
  sums over n tokens on the tensor cores, sixteen a step: (n / 16 + 32) * 2^-23, and as many roundings of the sum of the weights;
  the output's own rounding: 2^-11 of it, or 2^-25.
  |out - ref| <= 2^-11 |ref| + (2^-11 + 2 e_s + 2 (n / 16 + 32) 2^-23) sum p |v| + 2^-32 sum |v| + 2^-32 max (p 2^e) sum |code| + 2^-25
  |lse - ref| <= e_s + (n / 16 + 32) 2^-23 + 2^-22 |ref| + 2^-20.
"""
import ctypes
import math

import numpy as np
import pytest

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
            assert call(**{**base, name: base[name] + 2}) == ALIGN, name
            assert call(**{**base, name: None}) == (GONE if name in null else INV), name
        for bad in invalid:
            assert call(**{**base, **bad}) == INV, bad
        return base

    def cache(k, v, ks, vs, heads=2, page=16, pages=8):
        return ctypes.byref(B.Paged8Cache(k, v, ks, vs, pages, heads, page))

    rope = B.ecco_rope_init(64, np.ones(32))
    broken = [B.Rope.from_buffer_copy(rope) for _ in range(3)]
    broken[0].rot_dim, broken[1].gain, broken[2].flags = 8, math.inf, 16

    def append(kx, vx, slots, pos, stride=256, n=3, r=rope, **c):
        return L.ecco_paged8_append(cache(**c), ctypes.byref(r) if r is not None else None, pos, kx, vx, stride, slots, n, None)

    pools = ("k", "v", "ks", "vs")
    pages = (dict(page=0), dict(page=-16), dict(page=12), dict(page=8192), dict(pages=0), dict(pages=-1), dict(page=4096, pages=1 << 19))
    caches = pages + (dict(heads=0), dict(heads=-1), dict(heads=65536, stride=1 << 30))
    p = check(append, pools + ("kx", "vx", "slots", "pos"), caches + (dict(stride=248), dict(stride=-256), dict(stride=1 << 38), dict(n=-1), *(dict(r=r) for r in broken)))
    assert append(**p | {"stride": 260}) == ALIGN and append(**p | {"n": 0}) == 0 and append(**p | {"pos": None, "r": None}) == GONE and append(**p | {"pos": 3, "r": None}) == GONE
    for largest in (dict(heads=65535, stride=65535 * 128), dict(n=2**31 - 1), dict(stride=(1 << 38) - 8), dict(page=4096, pages=(1 << 19) - 1), dict(page=1, pages=2**31 - 1)):
        assert append(**p | largest) == GONE, largest
    for name in ("k", "v", "kx", "vx"):
        assert append(**p | {name: p[name] + 8}) == ALIGN and append(**p | {name: p[name] + 16}) == GONE, name
    assert L.ecco_paged8_append(None, None, None, 64, 128, 256, 192, 3, None) == INV

    def attn(tables, cu, lens, tiles, q, out, lse, ws, t_stride=4, n_req=2, tokens=3, new=2, kv=60, n_tiles=4, g=2, stride=512, scale=0.1, flags=1,
             ws_bytes=1 << 30, **c):
        b = B.PagedBatch(tables, cu, lens, tiles, t_stride, n_req, tokens, new, kv, n_tiles)
        return L.ecco_paged8_attn(cache(**c), ctypes.byref(b), g, q, stride, ctypes.c_float(scale), flags, out, lse, ws, ws_bytes, None)

    arrays = ("tables", "cu", "lens", "tiles", "q", "out", "lse")
    p = check(lambda **a: attn(ws=1 << 20, **a), pools + arrays, caches + (
        dict(g=0), dict(g=-1), dict(g=17, stride=1 << 20), dict(scale=math.nan), dict(scale=math.inf), dict(scale=-math.inf), dict(scale=3e38), dict(flags=2), dict(flags=3), dict(flags=1 << 31),
        dict(stride=504), dict(stride=-512), dict(stride=1 << 38), dict(t_stride=-1), dict(n_req=-1), dict(n_req=65536), dict(tokens=-1), dict(new=-1), dict(kv=-1),
        dict(n_tiles=-1), dict(n_tiles=1 << 25, heads=64, stride=1 << 20), dict(n_tiles=1 << 26, heads=1), dict(heads=4096, g=16, stride=1 << 30), dict(tokens=1 << 29),
        dict(tokens=1 << 26, kv=1 << 26)), null=("lse",))
    p["ws"] = 1 << 20
    for name in ("q", "out", "k", "v"):
        assert attn(**p | {name: p[name] + 8}) == ALIGN, name
    assert attn(**p | {"stride": 516}) == ALIGN
    for a, b in (("out", "q"), ("out", "ws"), ("q", "ws")):
        assert attn(**p | {a: p[b]}) == INV, (a, b)
    for fine in (dict(g=1), dict(g=16, stride=4096), dict(scale=0.0), dict(scale=-2.0), dict(scale=2e38), dict(flags=0), dict(t_stride=0, tables=None), dict(n_req=65535),
                 dict(stride=(1 << 38) - 8), dict(new=0), dict(kv=0), dict(n_tiles=0), dict(tokens=1 << 20, kv=1 << 20), dict(n_tiles=1 << 20)):
        assert attn(**p | fine) == GONE, fine
    assert attn(**p | {"n_req": 0}) == 0 and attn(**p | {"tokens": 0}) == 0
    batch = B.PagedBatch(64, 128, 192, 256, 4, 2, 3, 2, 60, 4)
    c = cache(4096, 8192, 12288, 16384)
    assert L.ecco_paged8_attn(None, ctypes.byref(batch), 2, 512, 512, ctypes.c_float(0.1), 1, 1024, None, 2048, 1 << 30, None) == INV
    assert L.ecco_paged8_attn(c, None, 2, 512, 512, ctypes.c_float(0.1), 1, 1024, None, 2048, 1 << 30, None) == INV
    need = lambda heads, new, g: int(L.ecco_paged8_attn_workspace_bytes(cache(64, 64, 64, 64, heads), ctypes.byref(B.PagedBatch(64, 64, 64, 64, 4, 2, 99, new, 6000, 400)), g))  # noqa: E731
    assert need(2, 1, 0) == 0 and 0 < need(2, 1, 1) < need(2, 90, 16) < 1 << 27 and need(2, 145, 16) >= need(2, 90, 16) + 400 * 2 * 2 * 8192
    assert need(0, 1, 1) == 0 and L.ecco_paged8_attn_workspace_bytes(None, ctypes.byref(batch), 2) == 0 and L.ecco_paged8_attn_workspace_bytes(c, None, 2) == 0


# ------------------------------------------------------------------ the format
CODES = np.array([(m * 2.0**-9 if e == 0 else (8 + m) * 2.0 ** (e - 10)) for e in range(16) for m in range(8)])
VALUES = np.concatenate([CODES, -CODES])                   # of a byte; 127 and 255, which nothing is rounded to, as 480
VALUES[[127, 255]] = [480, -480]


def nearest_code(x):
    """The E4M3 byte of an fp64 number: nearest, ties to even, saturating at 448."""
    x = np.asarray(x, np.float64)
    size = np.minimum(np.abs(x), 448.0)
    up = np.searchsorted(CODES[:127], size, side="left").clip(0, 126)
    down = np.maximum(up - 1, 0)
    gap_up, gap_down = CODES[up] - size, size - CODES[down]
    pick = np.where((gap_up < gap_down) | ((gap_up == gap_down) & (up % 2 == 0)), up, down)
    return (pick + 128 * np.signbit(x)).astype(np.uint8)


def power_of(top):
    """The smallest e in -15 .. 7 with top <= 448 * 2^e."""
    for e in range(-15, 8):
        if top <= 448 * 2.0**e:
            return e
    return 7


def append_reference(codes, scales, x, slots, page):
    """codes [pages][heads][page][128], scales [pages][heads][blocks] in place; x fp16 [tokens][heads][128], as it goes in."""
    places = min(16, page)
    x = np.where(np.isnan(x), 0, x).astype(np.float64)
    runs = {}
    for i, s in enumerate(slots):
        if 0 <= s < codes.shape[0] * page:
            runs.setdefault(s // places, []).append((i, s % places))
    for block, tokens in runs.items():
        at, nth = block * places // page, block * places % page // places
        for h in range(codes.shape[1]):
            e = power_of(max(np.abs(x[i, h]).max() for i, _ in tokens))
            here = codes[at, h, nth * places:(nth + 1) * places]
            if min(p for _, p in tokens) > 0:
                old = min(max(int(scales[at, h, nth]) - 127, -15), 7)
                e = max(e, old)
                if e > old:
                    for p in set(range(places)) - {p for _, p in tokens}:
                        here[p] = nearest_code(VALUES[here[p]] * 2.0 ** (old - e))
            for i, p in tokens:
                here[p] = nearest_code(x[i, h] * 2.0**-e)
            scales[at, h, nth] = e + 127


def random_rows(rng, shape, spread=4):
    x = rng.standard_normal(shape) * 10.0 ** rng.uniform(-spread, spread / 2, shape[:-1] + (1,))
    return x.clip(-65504, 65504).astype(np.float16)


def old_pool(rng, pages, heads, page):
    codes = rng.integers(0, 256, (pages, heads, page, 128)).astype(np.uint8)
    codes[(codes & 127) == 127] -= 1
    return codes, rng.integers(112, 135, (pages, heads, max(1, page // 16))).astype(np.uint8)


def run_append(B, pools, page, k, v, slots, rope=None, positions=None, stride=None, offset=0):
    """pools: [codes, scales] of K and of V; returns what they become.  k, v: fp16 [tokens][heads][128]."""
    pages, heads = pools[0][0].shape[:2]
    dev = [torch.from_numpy(np.concatenate([np.full(64, 165, np.uint8), a.reshape(-1), np.full(64, 90, np.uint8)])).cuda() for kind in pools for a in kind]
    kc, ks, vc, vs = (d.data_ptr() + 64 for d in dev)
    tokens = len(slots)
    stride = stride or heads * 128
    rows = torch.zeros((2, tokens, stride), dtype=torch.float16, device="cuda")
    for i, x in enumerate((k, v)):
        rows[i, :, offset:offset + heads * 128] = torch.from_numpy(x.reshape(tokens, -1)).cuda()
    cache = B.paged8_cache(kc, vc, ks, vs, pages, heads, page)
    B.ecco_paged8_append(cache, rope, ints(positions) if positions is not None else None, rows.data_ptr() + 2 * offset, rows[1].data_ptr() + 2 * offset, stride, ints(slots), tokens)
    torch.cuda.synchronize()
    got = [d.cpu().numpy() for d in dev]
    for g in got:
        assert (g[:64] == 165).all() and (g[-64:] == 90).all()
    flat = [g[64:-64] for g in got]
    return [[flat[2 * i].reshape(pools[i][0].shape), flat[2 * i + 1].reshape(pools[i][1].shape)] for i in range(2)]


def request_slots(rng, ctx, new, page, spare=2):
    """Slots of the new tokens of requests whose pages lie anywhere."""
    need = [-(-(c + n) // page) for c, n in zip(ctx, new)]
    order = rng.permutation(sum(need) + spare)
    slots, at = [], 0
    for c, n, m in zip(ctx, new, need):
        slots += [int(order[at + t // page]) * page + t % page for t in range(c, c + n)]
        at += m
    return slots, len(order)


@pytest.mark.gpu
@pytest.mark.parametrize("page", [1, 2, 8, 16, 32, 128, 4096])
@pytest.mark.parametrize("heads,requests,max_ctx,max_new", [(1, 1, 0, 1), (2, 5, 40, 1), (8, 3, 70, 60), (3, 40, 17, 3), (32, 2, 3, 33)])
def test_append_matches_the_definition(B, dev, page, heads, requests, max_ctx, max_new):
    if page == 4096 and heads > 8:
        requests = 1
    rng = np.random.default_rng([page, heads, requests])
    ctx, new = rng.integers(0, max_ctx + 1, requests), rng.integers(1, max_new + 1, requests)
    slots, pages = request_slots(rng, ctx, new, page)
    slots = slots + [-1] * int(rng.integers(0, 20))
    k, v = (random_rows(rng, (len(slots), heads, 128)) for _ in range(2))
    pools = [old_pool(rng, pages, heads, page) for _ in range(2)]
    want = [[a.copy() for a in kind] for kind in pools]
    for w, x in zip(want, (k, v)):
        append_reference(*w, x, slots, page)
    got = run_append(B, pools, page, k, v, slots, stride=heads * 128 + 24, offset=8)
    for w, g in zip(want, got):
        assert np.array_equal(w[1], g[1]) and np.array_equal(w[0], g[0])


@pytest.mark.gpu
def test_append_token_by_token(B, dev):
    """A request that grows a token at a time: the block's power of two follows its largest value, and begins anew with the block."""
    rng = np.random.default_rng(12)
    page, heads = 32, 2
    pools = [old_pool(rng, 3, heads, page) for _ in range(2)]
    want = [[a.copy() for a in kind] for kind in pools]
    for t in range(70):
        k, v = (random_rows(rng, (1, heads, 128), spread=3) for _ in range(2))
        slot = [(2, 0, 1)[t // page] * page + t % page]
        for w, x in zip(want, (k, v)):
            append_reference(*w, x, slot, page)
        pools = run_append(B, pools, page, k, v, slot)
        for w, g in zip(want, pools):
            assert np.array_equal(w[1], g[1]) and np.array_equal(w[0], g[0]), t


@pytest.mark.gpu
def test_append_values_at_the_borders(B, dev):
    """Values that saturate, vanish, tie and are not finite; largest values on both sides of 448 times a power of two."""
    tokens = []
    for e in range(-24, 16):
        for m in (1.0, 1.0625, 1.125, 1.74902, 1.75, 1.750977, 1.875, 1.9990234):
            x = np.zeros(128)
            x[:9] = m * 2.0**e * np.array([1, -1, 2.0**-3, 2.0**-7, 2.0**-8, 2.0**-14, 1.0625 / 2, 1.1875 / 4, 1.3125 / 8])
            tokens.append(x)
    tokens += [np.zeros(128), np.full(128, -0.0), np.full(128, np.nan), np.full(128, np.inf), np.r_[np.nan, np.ones(127)], np.r_[-np.inf, np.ones(127)],
               np.r_[57344.0, -57345.0, 65504.0, np.zeros(125)], np.full(128, 2.0**-24)]
    with np.errstate(over="ignore"):
        x = np.array(tokens).astype(np.float16)[:, None]
    for page in (1, 16):
        n = -(-len(x) // page) * page
        rng = np.random.default_rng(page)
        pools = [old_pool(rng, n // page, 1, page) for _ in range(2)]
        for slots in (list(range(len(x))), [s if s % 16 else -1 for s in range(len(x))]):            # blocks begun, and blocks that have a first token
            want = [[a.copy() for a in kind] for kind in pools]
            for w in want:
                append_reference(*w, x, slots, page)
            for w, g in zip(want, run_append(B, pools, page, x, x, slots)):
                assert np.array_equal(w[1], g[1]) and np.array_equal(w[0], g[0])


@pytest.mark.gpu
@pytest.mark.parametrize("rot,flags", [(128, 0), (128, 1), (64, 1), (48, 0), (16, 3), (112, 2)])
def test_append_turns_k_as_ecco_rope_apply_does(B, dev, rot, flags):
    rng = np.random.default_rng([rot, flags])
    page, heads = 16, 3
    ctx, new = rng.integers(0, 50, 9), rng.integers(1, 40, 9)
    slots, pages = request_slots(rng, ctx, new, page)
    slots += [-1, pages * page, 2**31 - 1, -7]
    k, v = (random_rows(rng, (len(slots), heads, 128), 2) for _ in range(2))
    positions = rng.integers(-100, 200000, len(slots))
    rope = B.ecco_rope_init(rot, 10000.0 ** (-np.arange(rot // 2) * 2 / rot), 0.9, flags)
    turned = torch.empty(k.shape, dtype=torch.float16, device="cuda")
    B.ecco_rope_apply(rope, ints(positions), len(slots), heads, torch.from_numpy(k).cuda(), heads * 128, turned, heads * 128)
    pools = [old_pool(rng, pages, heads, page) for _ in range(2)]
    want = [[a.copy() for a in kind] for kind in pools]
    for w, x in zip(want, (turned.cpu().numpy(), v)):
        append_reference(*w, x, slots, page)
    for w, g in zip(want, run_append(B, pools, page, k, v, slots, rope, positions)):
        assert np.array_equal(w[1], g[1]) and np.array_equal(w[0], g[0])


@pytest.mark.gpu
def test_append_whatever_the_slots(B, dev):
    """Slots in any order, several times the same, beyond the pool: what no slot names stays as it is, and so does what lies beside the pools."""
    rng = np.random.default_rng(14)
    for page in (4, 16, 64):
        for _ in range(4):
            tokens, heads, pages = int(rng.integers(1, 300)), 2, 12
            slots = rng.integers(-20, pages * page + 20, tokens)
            slots[rng.random(tokens) < 0.3] = int(rng.integers(0, pages * page))
            pools = [old_pool(rng, pages, heads, page) for _ in range(2)]
            x = random_rows(rng, (tokens, heads, 128))
            got = run_append(B, pools, page, x, x, slots)
            places = min(16, page)
            named = {int(s) // places for s in slots if 0 <= s < pages * page}
            for (codes, scales), (gc, gs) in zip(pools, got):
                for b in set(range(pages * page // places)) - named:
                    at, nth = b * places // page, b * places % page // places
                    assert np.array_equal(codes[at, :, nth * places:(nth + 1) * places], gc[at, :, nth * places:(nth + 1) * places])
                    assert np.array_equal(scales[at, :, nth], gs[at, :, nth])


# ------------------------------------------------------------------ attention
class Case:
    """Requests over pages anywhere in a pool of random blocks, padded rows behind them."""

    def __init__(self, B, rng, new, kv, heads, g, page, padding=3, qscale=1.0, spare=3, exps=(-9, -4)):
        self.B, self.new, self.kv, self.heads, self.g, self.page = B, list(map(int, new)), list(map(int, kv)), heads, g, page
        held = [-(-n // page) for n in self.kv]
        self.pages = sum(held) + spare
        order = rng.permutation(self.pages)
        self.stride = max(held + [0]) + 1
        tables = rng.integers(-9, 1 << 30, (len(new), self.stride)).astype(np.int32)       # what is not the request's is arbitrary
        at = 0
        for r, h in enumerate(held):
            tables[r, :h] = order[at:at + h]
            at += h
        self.tables = tables
        gen = torch.Generator(device="cuda").manual_seed(int(rng.integers(1 << 30)))
        self.pools = []
        for _ in range(2):
            codes = torch.randint(0, 256, (self.pages, heads, page, 128), generator=gen, device="cuda", dtype=torch.uint8)
            big = (codes & 127) >= 0x68                    # 16 and more: rarely, as channels that stick out
            codes = torch.where(big & (torch.rand(codes.shape, generator=gen, device="cuda") < 0.97), codes & 0xbf, codes)
            codes = torch.where((codes & 127) == 127, codes - 1, codes)
            # places behind a request's last token and pages of nobody hold anything, NaN among it
            scales = torch.randint(exps[0] + 127, exps[1] + 128, (self.pages, heads, max(1, page // 16)), generator=gen, device="cuda", dtype=torch.uint8)
            self.pools += [codes, scales]
        for r, n in enumerate(self.kv):
            if n % page:
                for i in (0, 2):
                    self.pools[i][int(tables[r, n // page]), :, n % page:] = 127 if i else 255
        self.tokens = sum(self.new) + padding
        self.padding = padding
        self.cu = np.concatenate([[0], np.cumsum(self.new)])
        self.tiles = np.concatenate([[0], np.cumsum([-(-n // 32) for n in self.kv])])
        self.q = (torch.randn((self.tokens, heads * g, 128), generator=gen, device="cuda") * qscale).half()
        self.cache = B.paged8_cache(self.pools[0], self.pools[2], self.pools[1], self.pools[3], self.pages, heads, page)
        self.arrays = [ints(tables), ints(self.cu), ints(self.kv), ints(self.tiles)]
        self.batch = self.make_batch(*self.arrays)

    def make_batch(self, tables, cu, kv, tiles, tokens=None, max_new=None, max_kv=None, max_tiles=None):
        pick = lambda a, b: b if a is None else a  # noqa: E731
        return self.B.paged_batch(tables, self.stride, cu, kv, tiles, len(self.new), pick(tokens, self.tokens), pick(max_new, max(self.new + [0])), pick(max_kv, max(self.kv + [0])),
                                  pick(max_tiles, int(self.tiles[-1])))

    def need(self, batch=None):
        return self.B.ecco_paged8_attn_workspace_bytes(self.cache, batch or self.batch, self.g)

    def run(self, causal=True, scale=128**-0.5, lse=True, ws_bytes=None, q=None, q_stride=None, batch=None, stream=None, ws=None):
        B, row = self.B, self.heads * self.g * 128
        out = torch.full((self.tokens, self.heads * self.g, 128), 7.0, dtype=torch.float16, device="cuda")
        d_lse = torch.full((self.tokens, self.heads * self.g), 7.0, device="cuda") if lse else None
        n = ws_bytes or self.need(batch)
        if ws is None:
            ws = torch.full((n + 256,), 0xa5, dtype=torch.uint8, device="cuda")
        B.ecco_paged8_attn(self.cache, batch or self.batch, self.g, self.q if q is None else q, q_stride or row, scale, B.ATTN_CAUSAL if causal else 0, out, d_lse, ws, n, stream=stream)
        torch.cuda.synchronize()
        if len(ws) > n:
            assert bool((ws[n:] == 0xa5).all())
        assert bool((out[self.tokens - self.padding:] == 7).all()) and (not lse or bool((d_lse[self.tokens - self.padding:] == 7).all()))
        return out, d_lse

    def values(self, r, h):
        """codes and powers of two of a request's tokens for a KV head, fp64."""
        n, page = self.kv[r], self.page
        t = torch.arange(n, device="cuda")
        at, place = torch.from_numpy(self.tables[r].astype(np.int64)).cuda()[t // page], t % page
        table = torch.from_numpy(VALUES).cuda()
        return [(table[self.pools[i][at, h, place].long()], torch.exp2(self.pools[i + 1][at, h, place // 16].double().clamp(112, 134) - 127)) for i in (0, 2)]

    def check(self, out, lse, causal=True, scale=128**-0.5, requests=None, q=None):
        q = self.q if q is None else q
        assert self.B.ecco_device_status() == 0
        for r in range(len(self.new)) if requests is None else requests:
            new, n = self.new[r], self.kv[r]
            rows = slice(int(self.cu[r]), int(self.cu[r]) + new)
            if new == 0:
                continue
            seen = (torch.arange(n, device="cuda")[None] < (n - new + 1 + torch.arange(new, device="cuda"))[:, None]) if causal else torch.ones((new, n), dtype=torch.bool, device="cuda")
            for hq in range(self.heads * self.g):
                got = out[rows, hq].double()
                if n == 0:
                    assert not got.any() and (lse is None or bool((lse[rows, hq] == -math.inf).all()))
                    continue
                (kc, ke), (vc, ve) = self.values(r, hq // self.g)
                k, v = kc * ke[:, None], vc * ve[:, None]
                x = q[rows, hq].double()
                s = (x @ k.T) * scale
                reach = ((x.abs() @ k.abs().T) * abs(scale)).where(seen, 0.0).amax(1)
                big = s.abs().where(seen, 0.0).amax(1)
                s = s.where(seen, -math.inf)
                ref_lse = s.logsumexp(1)
                p = (s - ref_lse[:, None]).exp().nan_to_num(0.0)
                ref = p @ v
                e_s = 128 * 2.0**-23 * reach + 2.0**-22 * (big + 23)
                steps = (n / 16 + 32) * 2.0**-23
                tol = 2.0**-11 * ref.abs() + (2.0**-11 + 2 * e_s + 2 * steps)[:, None] * (p @ v.abs()) + 2.0**-25
                tol += 2.0**-32 * (seen.double() @ v.abs()) + 2.0**-32 * (p * ve).amax(1)[:, None] * (seen.double() @ vc.abs())
                assert bool(((got - ref).abs() <= tol).all()), (r, hq, float(((got - ref).abs() / tol).max()))
                blind = ~seen.any(1)
                assert not got[blind].any()
                if lse is not None:
                    l = lse[rows, hq].double()
                    assert bool((l[blind] == -math.inf).all())
                    assert bool(((l - ref_lse).abs() <= e_s + steps + 2.0**-22 * ref_lse.abs() + 2.0**-20)[~blind].all())


SHAPES = [
    # new tokens, lengths, KV heads, query heads to one, page
    ([1], [1], 1, 1, 16), ([1], [31], 2, 4, 16), ([1, 1], [32, 33], 1, 8, 1), ([1] * 5, [0, 1, 100, 64, 7], 2, 3, 8), ([1] * 3, [2000, 5, 900], 8, 4, 16),
    ([1] * 2, [5000, 4999], 3, 1, 128), ([2, 8, 1], [300, 8, 77], 2, 1, 2), ([9, 3, 1, 0], [50, 1000, 65, 40], 2, 1, 32), ([1] * 4, [513, 1024, 31, 3], 1, 16, 4),
    ([4, 3, 8], [600, 3, 2500], 2, 4, 16), ([16, 15], [100, 500], 1, 4, 64), ([13, 1], [700, 700], 2, 5, 16), ([17, 1, 40], [64, 300, 41], 2, 4, 16),
    ([100, 1, 1], [1500, 900, 2], 2, 2, 8), ([300, 5, 0, 64], [300, 800, 10, 130], 1, 8, 4096), ([65], [65], 3, 1, 1), ([129, 2, 70], [200, 2000, 700], 2, 16, 32),
    ([1] * 300, [37] * 300, 1, 2, 16), ([1] * 40, list(range(0, 400, 10)), 4, 4, 16),
    # enough tiles for the kernel of many rows
    ([300, 5, 0, 64], [3000, 800, 10, 130], 2, 8, 16), ([130, 1, 1], [1500, 900, 2], 8, 3, 8), ([400, 33], [400, 2000], 2, 16, 128), ([70, 70, 1], [4000, 69, 31], 3, 16, 4),
    ([1000], [1000], 4, 2, 32), ([257, 1, 300], [5000, 0, 257], 1, 13, 1), ([515, 20], [20, 515], 6, 4, 64),
]


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "%dx%d-%d_%dx%d_p%d" % (len(s[0]), max(s[0]), max(s[1]), s[2], s[3], s[4]))
def test_attention(B, dev, shape, causal):
    new, kv, heads, g, page = shape
    c = Case(B, np.random.default_rng([len(new), sum(kv), heads, g, page]), new, kv, heads, g, page)
    out, lse = c.run(causal)
    c.check(out, lse, causal)
    again, lse_again = c.run(causal)                       # the order of the sums is that of the batch
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and torch.equal(lse.view(torch.int32), lse_again.view(torch.int32))
    alone, _ = c.run(causal, lse=False)
    assert torch.equal(out.view(torch.int16), alone.view(torch.int16))


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [0.0, -0.1, 1e-4, 3.0])
@pytest.mark.parametrize("new", [1, 40, 300])
def test_scales(B, dev, scale, new):
    c = Case(B, np.random.default_rng([new]), [new, 2], [400, 90], 2 if new < 300 else 16, 4, 16)
    out, lse = c.run(scale=scale)
    c.check(out, lse, scale=scale)


@pytest.mark.gpu
@pytest.mark.parametrize("new", [1, 5, 60, 300])
def test_powers_of_two_of_all_sizes(B, dev, new):
    """Blocks of 2^-15 beside blocks of 2^7: the weights of the first are not lost beside the second's."""
    c = Case(B, np.random.default_rng([new, 7]), [new, new], [700, 130], 2 if new < 300 else 8, 3, 16, qscale=2.0**-7, exps=(-15, 7))
    out, lse = c.run()
    c.check(out, lse)
    # V of the smallest power of two where K draws the weight, of the largest where it does not
    c.pools[3][:] = 112
    c.pools[3][::2] = 134
    c.pools[1][:] = 117
    out, lse = c.run()
    c.check(out, lse)
    # bytes that are no power of two of this cache count as the nearest of them
    c.pools[3][:] = torch.where(c.pools[3] == 112, 0, 255).to(torch.uint8)
    again, lse_again = c.run()
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and torch.equal(lse, lse_again)


@pytest.mark.gpu
@pytest.mark.parametrize("new", [[3, 1], [70, 1], [9, 4], [900, 900]])
def test_more_new_tokens_than_the_request_holds(B, dev, new):
    """The first rows of such a request see nothing: zeros, and minus infinity."""
    kv, heads = [2, 0], 2
    if new[0] == 900:                                      # the tiles of another request make it a call for the kernel of many rows
        new, kv, heads = new + [1], kv + [900], 8
    c = Case(B, np.random.default_rng(new), new, kv, heads, 2, 16)
    out, lse = c.run()
    c.check(out, lse)
    assert not out[:new[0] - 2].any() and bool((lse[:new[0] - 2] == -math.inf).all())


@pytest.mark.gpu
@pytest.mark.parametrize("new", [1, 30, 300])
def test_q_that_is_not_finite_spoils_its_own_rows(B, dev, new):
    c = Case(B, np.random.default_rng([new, 5]), [new, new], [max(200, new), max(64, new)], 2 if new < 300 else 16, 4, 16)
    clean, clean_lse = c.run()
    q = c.q.clone()
    q[0, 1, 5], q[new, 6, 0] = math.nan, math.inf
    out, lse = c.run(q=q)
    bad = torch.zeros(c.q.shape[:2], dtype=torch.bool, device="cuda")
    bad[0, 1] = bad[new, 6] = True
    assert bool(out[0, 1].isnan().all()) and bool(lse[0, 1].isnan())
    assert torch.equal(out[~bad].view(torch.int16), clean[~bad].view(torch.int16)) and torch.equal(lse[~bad], clean_lse[~bad])


@pytest.mark.gpu
def test_strided_q_and_no_workspace(B, dev):
    for new, kv in (([1, 3], [300, 70]), ([50, 1, 70], [400, 300, 70]), ([500, 1], [3000, 70])):
        c = Case(B, np.random.default_rng(new), new, kv, 4, 4, 16)
        out, lse = c.run()
        c.check(out, lse)
        wide = torch.full((c.tokens, c.heads * c.g * 128 + 256 + 8), float("nan"), dtype=torch.float16, device="cuda")
        wide[:, :c.heads * c.g * 128] = c.q.reshape(c.tokens, -1)
        again, _ = c.run(q=wide, q_stride=wide.shape[1])
        assert torch.equal(out.view(torch.int16), again.view(torch.int16))
        with pytest.raises(B.EccoError) as e:
            c.run(ws_bytes=256)
        assert e.value.code == B.ERR_WORKSPACE
        with pytest.raises(B.EccoError) as e:
            B.ecco_paged8_attn(c.cache, c.batch, c.g, c.q, c.heads * c.g * 128, 0.1, 0, torch.empty_like(c.q), None, None, 1 << 30)
        assert e.value.code == B.ERR_WORKSPACE


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("page", [1, 4, 16, 64, 256])
def test_a_long_prompt_with_and_without_room_for_its_tiles(B, dev, page, causal):
    """2304 rows of a request are the last for which no tiles are made beforehand, where there is room for them."""
    c = Case(B, np.random.default_rng([page, causal]), [288, 289, 1, 577], [1000, 289, 130, 700], 2, 8, page)
    least = int(B.lib().ecco_paged8_attn_workspace_bytes(ctypes.byref(c.cache), ctypes.byref(c.make_batch(*c.arrays, max_tiles=0)), c.g))
    assert least < c.need() == int(B.lib().ecco_paged8_attn_workspace_bytes(ctypes.byref(c.cache), ctypes.byref(c.batch), c.g))
    for n in (c.need(), c.need() - 1, least):
        out, lse = c.run(causal, ws_bytes=n)
        c.check(out, lse, causal)
    with pytest.raises(B.EccoError) as e:
        c.run(causal, ws_bytes=least // 4)             # the sizes are for up to 256 SMs
    assert e.value.code == B.ERR_WORKSPACE


@pytest.mark.gpu
@pytest.mark.parametrize("new", [1, 70, 300])
def test_more_requests_than_fit_shared_memory(B, dev, new):
    rng = np.random.default_rng([new, 11])
    n = 1500
    news = rng.integers(0, 3, n)
    news[[3, 1200]] = new
    c = Case(B, rng, news, rng.integers(0, 80, n), 1, 2, 16)
    out, lse = c.run()
    c.check(out, lse, requests=[0, 1, 2, 3, 700, 701, 702, 703, 1199, 1200, 1201, 1499])
    for r in range(n):                                     # rows that see nothing
        if c.kv[r] == 0 and c.new[r]:
            rows = slice(int(c.cu[r]), int(c.cu[r + 1]))
            assert not out[rows].any() and bool((lse[rows] == -math.inf).all()), r


@pytest.mark.gpu
def test_a_long_request_alone(B, dev):
    """One request and head over the whole machine, and the join of all its pieces."""
    for new, g in ((1, 1), (1, 16), (6, 8)):
        c = Case(B, np.random.default_rng([new, g]), [new], [60001], 1, g, 64)
        out, lse = c.run()
        c.check(out, lse)


@pytest.mark.gpu
def test_captured_and_replayed_with_other_lengths(B, dev):
    """The sizes that the host passes are upper bounds; two graphs share a workspace."""
    rng = np.random.default_rng(21)
    for max_new, g in ((1, 4), (40, 4), (200, 8)):
        cases = [Case(B, np.random.default_rng([s, max_new]), rng.integers(0, max_new + 1, 6), rng.integers(0, 900, 6), 2, g, 16, padding=0) for s in range(3)]
        bound = dict(tokens=6 * max_new, max_new=max_new, max_kv=1000, max_tiles=6 * 32)
        c = cases[0]
        stride = max(x.stride for x in cases)
        tables, cu, kv, tiles = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (6 * stride, 7, 6, 7))
        pools = [torch.zeros((max(x.pages for x in cases),) + tuple(p.shape[1:]), dtype=torch.uint8, device="cuda") for p in c.pools]
        cache = B.paged8_cache(pools[0], pools[2], pools[1], pools[3], len(pools[0]), 2, 16)
        batch = B.paged_batch(tables, stride, cu, kv, tiles, 6, 6 * max_new, bound["max_new"], bound["max_kv"], bound["max_tiles"])
        q = torch.zeros((6 * max_new, 2 * g, 128), dtype=torch.float16, device="cuda")
        n = B.ecco_paged8_attn_workspace_bytes(cache, batch, g)
        ws = torch.full((n,), 0x3c, dtype=torch.uint8, device="cuda")
        outs = [torch.zeros_like(q) for _ in range(2)]
        lses = [torch.zeros(q.shape[:2], device="cuda") for _ in range(2)]
        call = lambda i: B.ecco_paged8_attn(cache, batch, g, q, 2 * g * 128, 128**-0.5, B.ATTN_CAUSAL, outs[i], lses[i], ws, n)  # noqa: E731
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call(0)
        side.synchronize()
        graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
        for i, graph in enumerate(graphs):
            with torch.cuda.graph(graph):
                call(i)
        for turn in range(6):
            x = cases[turn % 3]
            padded = np.zeros((6, stride), np.int32)
            padded[:, :x.stride] = x.tables
            tables.copy_(ints(padded.reshape(-1)))
            cu.copy_(ints(x.cu)); kv.copy_(ints(x.kv)); tiles.copy_(ints(x.tiles))  # noqa: E702
            for dst, src in zip(pools, x.pools):
                dst[:len(src)] = src
            q[:x.tokens] = x.q
            for i in (0, 1):
                outs[i].fill_(7.0)
                graphs[i].replay()
            torch.cuda.synchronize()
            for i in (0, 1):
                x.check(outs[i], lses[i])
                assert bool((outs[i][x.tokens:] == 7).all())


@pytest.mark.gpu
def test_two_streams_at_once(B, dev):
    cases = [Case(B, np.random.default_rng([s, 3]), new, kv, 4, 4, 16) for s, (new, kv) in enumerate((([1] * 6, [900] * 6), ([40, 1, 1], [800, 700, 600]), ([300, 80], [900, 700])))]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    results = []
    for c, st in zip(cases, streams):
        out, lse = torch.zeros_like(c.q), torch.zeros(c.q.shape[:2], device="cuda")
        ws = torch.empty(c.need(), dtype=torch.uint8, device="cuda")
        results.append((out, lse, ws))
    torch.cuda.synchronize()
    for _ in range(20):
        for c, st, (out, lse, ws) in zip(cases, streams, results):
            B.ecco_paged8_attn(c.cache, c.batch, c.g, c.q, c.heads * c.g * 128, 128**-0.5, B.ATTN_CAUSAL, out, lse, ws, len(ws), stream=st)
    torch.cuda.synchronize()
    for c, (out, lse, _) in zip(cases, results):
        c.check(out, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("what", ["page", "no page", "falling", "negative", "too long", "too many", "more rows", "lengths", "beyond"])
@pytest.mark.parametrize("new", [1, 40, 600, 1200])
def test_wrong_arrays_are_reported(B, dev, what, new):
    """Arrays that say what cannot be: reported, nothing beside the buffers is touched, and the next call is what it always is."""
    c = Case(B, np.random.default_rng([new, 8]), [new, 1, 2], [150, 90, 33], 2 if new < 600 else 16, 4, 16)
    tables, cu, kv, tiles = c.tables.copy(), c.cu.copy(), np.array(c.kv), c.tiles.copy()
    bounds = {}
    if what == "page":
        tables[1, 2] = c.pages
    elif what == "no page":
        tables[0, 0] = -1
    elif what == "falling":
        tiles[2] = tiles[1] - 1
    elif what == "negative":
        tiles[1] = -4
    elif what == "too long":
        kv[1] = 32 * 5
    elif what == "too many":
        bounds["max_tiles"] = int(tiles[-1]) - 2
    elif what == "more rows":
        bounds["max_new"] = 1 if new > 1 else 0
    elif what == "lengths":
        kv[0] = -3
    elif what == "beyond":
        cu[3] = c.tokens + 50
    batch = c.make_batch(ints(tables), ints(cu), ints(kv), ints(tiles), **bounds)
    n = max(c.need(batch), c.need())
    guard = [torch.full((k,), 0x5a, dtype=torch.uint8, device="cuda") for k in (n + 512, c.tokens * c.heads * c.g * 256 + 512)]
    B.ecco_paged8_attn(c.cache, batch, c.g, c.q, c.heads * c.g * 128, 0.1, B.ATTN_CAUSAL, guard[1].data_ptr() + 256, None, guard[0].data_ptr() + 256, n)
    assert B.ecco_device_status() == B.ERR_INVALID_ARG
    for t in guard:
        assert bool((t[:256] == 0x5a).all()) and bool((t[-256:] == 0x5a).all())
    out, lse = c.run(ws=guard[0][256:-256].contiguous())
    c.check(out, lse)


@pytest.mark.gpu
def test_random_batches(B, dev):
    rng = np.random.default_rng(31)
    for _ in range(60):
        heads, g, page = int(rng.choice([1, 2, 3, 8])), int(rng.choice([1, 2, 3, 4, 5, 7, 8, 16])), int(rng.choice([1, 2, 4, 8, 16, 32, 64, 256]))
        n = int(rng.integers(1, 30))
        most = int(rng.choice([1, 1, 2, 5, 20, 150, 400]))
        new = rng.integers(0, most + 1, n)
        new[0] = max(new[0], 1)
        kv = (new * rng.integers(0, 2, n) + rng.integers(0, int(10 ** rng.uniform(0.5, 3.3)), n)).astype(int)
        if heads * g * new.sum() * kv.max() > 2e8:
            kv = kv // 8
        causal = bool(rng.integers(0, 2))
        c = Case(B, rng, new, kv, heads, g, page)
        out, lse = c.run(causal)
        c.check(out, lse, causal, requests=rng.choice(n, min(n, 4), replace=False))


# ------------------------------------------------------------------ as they are used together
@pytest.mark.gpu
@pytest.mark.parametrize("page,rot,flags", [(16, 128, 0), (64, 64, 1), (8, 32, 0)])
def test_steps_of_a_server(B, dev, page, rot, flags):
    """A prompt step, a mixed step and decode steps: ecco_paged_plan, ecco_rope_apply on the queries, ecco_paged8_append, ecco_paged8_attn; against plain
    attention in 64 bits over keys that are turned and values as they came, with the cache's rounding (2^-4 of each number, or half of the
    smallest step under its power of two) as tolerance."""
    rng = np.random.default_rng([page, rot])
    heads, g, n = 2, 4, 4
    scale = 128**-0.5
    f = 10000.0 ** (-np.arange(rot // 2) * 2 / rot)
    rope = B.ecco_rope_init(rot, f, flags=flags)
    stride, pages = 400 // page + 2, 4 * (400 // page + 2)
    codes = [torch.full((pages, heads, page, 128), 127, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.zeros((pages, heads, max(1, page // 16)), dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = B.paged8_cache(codes[0], codes[1], scales[0], scales[1], pages, heads, page)
    tables, free = torch.zeros((n, stride), dtype=torch.int32, device="cuda"), ints(rng.permutation(pages))
    taken, ctx = 0, np.zeros(n, int)
    history = [[] for _ in range(n)]                       # per request: rows of q, k, v
    for new in ([100, 5, 0, 37], [1, 64, 3, 1], [1, 1, 1, 1], [1, 1, 1, 1], [0, 0, 2, 1]):
        rows = sum(new)
        padded = rows + 5
        qkv = (rng.standard_normal((padded, heads * (g + 2), 128))).astype(np.float16)
        d = torch.from_numpy(qkv).cuda()
        row, at = heads * (g + 2) * 128, d.data_ptr()
        slots, cu, lens, tiles, result = (torch.zeros(k, dtype=torch.int32, device="cuda") for k in (padded, n + 1, n, n + 1, 4))
        B.ecco_paged_plan(page, pages, n, ints(ctx), ints(new), free[taken:], pages - taken, tables, stride, slots, padded, cu, lens, tiles, result)
        positions = np.concatenate([np.arange(c, c + k) for c, k in zip(ctx, new)] + [np.zeros(5, int)])
        B.ecco_rope_apply(rope, ints(positions), padded, heads * g, d, row, d, row)
        B.ecco_paged8_append(cache, rope, ints(positions), at + heads * g * 256, at + heads * (g + 1) * 256, row, slots, padded)
        bounds = (max(new), 400, n * 13)
        batch = B.paged_batch(tables, stride, cu, lens, tiles, n, padded, *bounds)
        ws = torch.empty(B.ecco_paged8_attn_workspace_bytes(cache, batch, g), dtype=torch.uint8, device="cuda")
        out = torch.full((padded, heads * g, 128), 7.0, dtype=torch.float16, device="cuda")
        B.ecco_paged8_attn(cache, batch, g, d, row, scale, B.ATTN_CAUSAL, out, None, ws, len(ws))
        taken += int(result[1])
        assert int(result[0]) == 0 and B.ecco_device_status() == 0 and bool((out[rows:] == 7).all())
        first = 0
        for r, k in enumerate(new):
            history[r] += list(qkv[first:first + k])
            ctx[r] += k
            if k:
                x = np.array(history[r]).astype(np.float64)
                turn = np.arange(len(x))[:, None] * f
                i = np.arange(rot // 2)
                a, b = (2 * i, 2 * i + 1) if flags else (i, i + rot // 2)
                y = x[:, :heads * (g + 1)].copy()
                y[..., a], y[..., b] = (x[:, :heads * (g + 1), a] * np.cos(turn)[:, None] - x[:, :heads * (g + 1), b] * np.sin(turn)[:, None],
                                        x[:, :heads * (g + 1), b] * np.cos(turn)[:, None] + x[:, :heads * (g + 1), a] * np.sin(turn)[:, None])
                for hq in range(heads * g):
                    q, key, v = y[-k:, hq], y[:, heads * g + hq // g], x[:, heads * (g + 1) + hq // g]
                    s = scale * q @ key.T
                    see = np.arange(len(x))[None] <= (len(x) - k + np.arange(k))[:, None]
                    # a key's value is off by 2^-4 of it, or, of a block whose largest is below 8 (four standard deviations and more), 2^-10 * 2^-5
                    # (the smallest e with 8 <= 448 * 2^e is -5): |s| by so much of sum |q k|; weights by e^that, either way; and the
                    # roundings of q to fp16 and of the kernel, which are small beside them
                    d_s = (scale * (np.abs(q) @ (np.abs(key) * 2.0**-4 + 2.0**-15).T) * 1.01 + 2e-3).max(1)
                    p = np.where(see, np.exp(s - s.max(1, keepdims=True)), 0)
                    p /= p.sum(1, keepdims=True)
                    got = out[first:first + k, hq].cpu().numpy().astype(np.float64)
                    tol = np.expm1(2 * d_s)[:, None] * (p @ np.abs(v)) * (1 + 2.0**-4) + p @ (np.abs(v) * 2.0**-4 + 2.0**-15) + 2e-3
                    assert np.all(np.abs(got - p @ v) <= tol)
            first += k


# ------------------------------------------------------------------ the far ends
@pytest.mark.gpu
def test_offsets_beyond_32_bits(B, dev):
    """Pools of 6.4 GB each: the last pages and the first."""
    rng = np.random.default_rng(41)
    page, heads, g, pages = 32, 2, 4, 780_000
    codes = [torch.empty((pages, heads, page, 128), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.empty((pages, heads, 2), dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = B.paged8_cache(codes[0], codes[1], scales[0], scales[1], pages, heads, page)
    kv, new = [100, 70, 33], [1, 70, 5]
    tables = np.array([[pages - 1, 0, pages - 2, 524_288], [pages - 3, 1, 655_360, -1], [2, pages - 4, -1, -1]], np.int32)
    rows = sum(kv)
    k, v = (rng.standard_normal((rows, heads, 128)).astype(np.float16) for _ in range(2))
    slots = [int(tables[r, t // page]) * page + t % page for r, n in enumerate(kv) for t in range(n)]
    d = torch.from_numpy(np.stack([k, v])).cuda()
    B.ecco_paged8_append(cache, None, None, d[0], d[1], heads * 128, ints(slots), rows)
    names = sorted({int(p) for r, n in enumerate(kv) for p in tables[r, :-(-n // page)]})
    local = [names.index(s // page) * page + s % page for s in slots]
    for i, x in enumerate((k, v)):
        want = np.zeros((len(names), heads, page, 128), np.uint8)
        append_reference(want, np.zeros((len(names), heads, 2), np.uint8), x, local, page)
        here = codes[i][torch.tensor(names, device="cuda")].cpu().numpy()
        taken = np.zeros((len(names), page), bool)
        for s in local:
            taken[s // page, s % page] = True
        assert np.array_equal(here.transpose(0, 2, 1, 3)[taken], want.transpose(0, 2, 1, 3)[taken])
    cu, tiles = np.concatenate([[0], np.cumsum(new)]), np.concatenate([[0], np.cumsum([-(-n // 32) for n in kv])])
    batch = B.paged_batch(ints(tables), 4, ints(cu), ints(kv), ints(tiles), 3, sum(new), max(new), max(kv), int(tiles[-1]))
    q = torch.from_numpy(rng.standard_normal((sum(new), heads * g, 128)).astype(np.float16)).cuda()
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
    ws = torch.empty(B.ecco_paged8_attn_workspace_bytes(cache, batch, g), dtype=torch.uint8, device="cuda")
    B.ecco_paged8_attn(cache, batch, g, q, heads * g * 128, 128**-0.5, B.ATTN_CAUSAL, out, lse, ws, len(ws))
    c = Case.__new__(Case)
    c.B, c.new, c.kv, c.heads, c.g, c.page, c.tables, c.cu, c.q = B, new, kv, heads, g, page, tables, cu, q
    c.pools = [codes[0], scales[0], codes[1], scales[1]]
    c.check(out, lse)


@pytest.mark.gpu
def test_a_replay_after_one_with_wrong_arrays(B, dev):
    """What a call with arrays that cannot be leaves in the workspace does not change what the same graph computes afterwards."""
    for new in (1, 40, 150):
        c = Case(B, np.random.default_rng([new, 51]), [new] * 5, [700, 650, 900, 40, 800], 4 if new < 150 else 8, 4, 16, padding=0)
        out, lse = torch.zeros_like(c.q), torch.zeros(c.q.shape[:2], device="cuda")
        ws = torch.empty(c.need(), dtype=torch.uint8, device="cuda")
        call = lambda: B.ecco_paged8_attn(c.cache, c.batch, c.g, c.q, c.heads * c.g * 128, 128**-0.5, B.ATTN_CAUSAL, out, lse, ws, len(ws))  # noqa: E731
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        good = [a.clone() for a in c.arrays]
        for which, at, value in ((3, 2, 0), (2, 1, 10_000), (1, 3, -5), (3, 5, 1 << 20), (0, 0, 1 << 30)):
            c.arrays[which].view(-1)[at] = value
            graph.replay()
            assert B.ecco_device_status() == B.ERR_INVALID_ARG, (which, at)
            c.arrays[which].copy_(good[which])
            out.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            c.check(out, lse)


@pytest.mark.gpu
def test_calls_behind_one_another(B, dev):
    """Turned, appended and attended to many times without a pause: each kernel begins while the one in front ends."""
    rng = np.random.default_rng(61)
    heads, g, page, n, steps = 2, 4, 16, 7, 40
    rope = B.ecco_rope_init(128, 10000.0 ** (-np.arange(64) / 64))
    stride, pages = 8, n * 8
    tables = np.arange(pages).reshape(n, stride)[:, ::-1].astype(np.int32).copy()
    qkv = rng.standard_normal((steps, n, heads * (g + 2), 128)).astype(np.float16)
    row = heads * (g + 2) * 128

    def serve(wait):
        codes = [torch.full((pages, heads, page, 128), 127, dtype=torch.uint8, device="cuda") for _ in range(2)]
        scales = [torch.zeros((pages, heads, 1), dtype=torch.uint8, device="cuda") for _ in range(2)]
        cache = B.paged8_cache(codes[0], codes[1], scales[0], scales[1], pages, heads, page)
        d, outs = torch.from_numpy(qkv).cuda(), []
        arrays = [[ints(tables), ints(np.arange(n + 1)), ints([s + 1] * n), ints(np.arange(n + 1) * (s // 32 + 1))] for s in range(steps)]
        slots = [ints([int(tables[r, s // page]) * page + s % page for r in range(n)]) for s in range(steps)]
        positions = [ints([s] * n) for s in range(steps)]
        batches = [B.paged_batch(a[0], stride, a[1], a[2], a[3], n, n, 1, steps, n * 2) for a in arrays]
        ws = torch.empty(B.ecco_paged8_attn_workspace_bytes(cache, batches[0], g), dtype=torch.uint8, device="cuda")
        outs = [torch.zeros((n, heads * g, 128), dtype=torch.float16, device="cuda") for _ in range(steps)]
        torch.cuda.synchronize()
        for s in range(steps):
            at = d[s].data_ptr()
            for call in (lambda: B.ecco_rope_apply(rope, positions[s], n, heads * g, d[s], row, d[s], row),
                         lambda: B.ecco_paged8_append(cache, rope, positions[s], at + heads * g * 256, at + heads * (g + 1) * 256, row, slots[s], n),
                         lambda: B.ecco_paged8_attn(cache, batches[s], g, d[s], row, 128**-0.5, B.ATTN_CAUSAL, outs[s], None, ws, len(ws))):
                call()
                if wait:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        return [*codes, *scales, *outs]

    for a, b in zip(serve(False), serve(True)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.gpu
@pytest.mark.parametrize("page", [4, 16])
def test_the_least_alignment(B, dev, page):
    """Pools, q, rows, out and workspace at odd multiples of 16 bytes, scales, lse and arrays at odd multiples of 4."""
    def at(t, off):
        d = torch.zeros(t.numel() * t.element_size() + 64, dtype=torch.uint8, device="cuda")
        assert d.data_ptr() % 64 == 0
        d[off:off + t.numel() * t.element_size()] = t.contiguous().view(-1).view(torch.uint8)
        return d, d.data_ptr() + off

    for new, kv, heads, g in (([1, 1], [300, 40], 2, 4), ([300, 30], [2000, 700], 4, 4), ([600, 30], [2000, 700], 2, 8)):
        c = Case(B, np.random.default_rng([page] + new), new, kv, heads, g, page)
        out, lse = c.run()
        keep = [at(t, off) for t, off in zip(c.pools, (16, 4, 48, 12))] + [at(t, 4) for t in c.arrays]
        q, o, l = at(c.q, 16), at(torch.full_like(out, 7.0), 48), at(torch.full_like(lse, 7.0), 4)
        ws = torch.zeros(c.need() + 64, dtype=torch.uint8, device="cuda")
        cache = B.paged8_cache(keep[0][1], keep[2][1], keep[1][1], keep[3][1], c.pages, heads, page)
        batch = B.paged_batch(keep[4][1], c.stride, keep[5][1], keep[6][1], keep[7][1], len(new), c.tokens, max(new), max(kv), int(c.tiles[-1]))
        B.ecco_paged8_attn(cache, batch, g, q[1], heads * g * 128, 128**-0.5, B.ATTN_CAUSAL, o[1], l[1], ws.data_ptr() + 16, c.need())
        torch.cuda.synchronize()
        c.check(o[0][48:48 + out.numel() * 2].view(torch.float16).view(out.shape), l[0][4:4 + lse.numel() * 4].view(torch.float32).view(lse.shape))
    rng = np.random.default_rng([page, 5])
    slots, pages = request_slots(rng, [3, 0, 20], [30, 70, 1], page)
    k, v = (random_rows(rng, (len(slots), 3, 128)) for _ in range(2))
    pools = [old_pool(rng, pages, 3, page) for _ in range(2)]
    want = [[a.copy() for a in kind] for kind in pools]
    for w, x in zip(want, (k, v)):
        append_reference(*w, x, slots, page)
    held = [at(torch.from_numpy(a), off) for a, off in zip([a for kind in pools for a in kind], (16, 4, 48, 12))]
    rows = [at(torch.from_numpy(x), 16) for x in (k, v)]
    index = at(ints(slots), 4)
    B.ecco_paged8_append(B.paged8_cache(held[0][1], held[2][1], held[1][1], held[3][1], pages, 3, page), None, None, rows[0][1], rows[1][1], 3 * 128, index[1], len(slots))
    torch.cuda.synchronize()
    for (d, _), off, w in zip(held, (16, 4, 48, 12), [a for kind in want for a in kind]):
        assert np.array_equal(d[off:off + w.size].cpu().numpy(), w.reshape(-1))


@pytest.mark.gpu
@pytest.mark.parametrize("new,kv", [([3, 1], [0, 0]), ([1, 2, 40], [0, 300, 90]), ([2, 700, 1], [2100, 700, 0])])
def test_the_largest_bounds(B, dev, new, kv):
    """Bounds far above what the arrays say, and of tiles none where there are none."""
    c = Case(B, np.random.default_rng(new), new, kv, 2, 16, 16)
    tiles = int(c.tiles[-1])
    for most in (dict(max_new=2**31 - 1, max_tiles=tiles), dict(max_new=2**31 - 1, max_tiles=tiles, max_kv=2**31 - 1 if c.tokens < 600 else 1 << 24), dict(max_new=2**31 - 1, max_tiles=tiles + 5000)):
        out, lse = c.run(batch=c.make_batch(*c.arrays, **most))
        c.check(out, lse)


@pytest.mark.gpu
def test_mixed_calls_behind_one_another(B, dev):
    """As above with a piece of a prompt beside single tokens in every step, so that the kernel for few rows begins while the one for many ends, right
    behind an append that has given the blocks in question other powers of two."""
    rng = np.random.default_rng(62)
    heads, g, page, n, piece, steps = 8, 4, 16, 24, 100, 24
    rope = B.ecco_rope_init(128, 10000.0 ** (-np.arange(64) / 64))
    ctx = np.r_[rng.integers(1, 400, n - 1), 1500]
    new = np.r_[np.ones(n - 1, int), piece]
    held = -(-(ctx + steps * new) // page)
    stride, pages, rows = int(held.max()), int(held.sum()), int(new.sum())
    order, tables = rng.permutation(pages), np.full((n, stride), -1, np.int32)
    for r, at in enumerate(np.cumsum(held) - held):
        tables[r, :held[r]] = order[at:at + held[r]]
    row = heads * (g + 2) * 128
    place = lambda r, t: [int(tables[r, i // page]) * page + i % page for i in t]  # noqa: E731
    start = torch.from_numpy(rng.standard_normal((int(ctx.sum()), heads * 2, 128)).astype(np.float16)).cuda()
    start_slots = ints([s for r in range(n) for s in place(r, range(ctx[r]))])
    # a step's K and V are up to twice as large as the step's before, sixteen steps long, then small again
    gen = torch.Generator(device="cuda").manual_seed(63)
    qkv = torch.randn((steps, rows, heads * (g + 2), 128), generator=gen, device="cuda")
    qkv[:, :, heads * g:] *= 2.0 ** (torch.arange(steps, device="cuda") % 16 - 8)[:, None, None, None]
    qkv = qkv.half()
    lens = [ctx + (s + 1) * new for s in range(steps)]
    tiles = [np.r_[0, np.cumsum(-(-x // 32))] for x in lens]
    tokens = [np.concatenate([np.arange(c, c + k) for c, k in zip(ctx + s * new, new)]) for s in range(steps)]
    slots = [ints([x for r in range(n) for x in place(r, range(ctx[r] + s * new[r], lens[s][r]))]) for s in range(steps)]
    positions, cu, d_tables = [ints(t) for t in tokens], ints(np.r_[0, np.cumsum(new)]), ints(tables)
    arrays = [(ints(x), ints(t)) for x, t in zip(lens, tiles)]
    batches = [B.paged_batch(d_tables, stride, cu, a, t, n, rows, piece, int(lens[-1].max()), int(tiles[-1][-1])) for a, t in arrays]

    def serve(wait):
        codes = [torch.full((pages, heads, page, 128), 127, dtype=torch.uint8, device="cuda") for _ in range(2)]
        scales = [torch.zeros((pages, heads, 1), dtype=torch.uint8, device="cuda") for _ in range(2)]
        cache = B.paged8_cache(codes[0], codes[1], scales[0], scales[1], pages, heads, page)
        B.ecco_paged8_append(cache, None, None, start, start.data_ptr() + heads * 256, heads * 256, start_slots, len(start))
        need = B.ecco_paged8_attn_workspace_bytes(cache, batches[0], g)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        d = qkv.clone()
        outs = [torch.zeros((rows, heads * g, 128), dtype=torch.float16, device="cuda") for _ in range(steps)]
        torch.cuda.synchronize()
        before = B.ecco_kernel_launch_count()
        for s in range(steps):
            at = d[s].data_ptr()
            for call in (lambda: B.ecco_rope_apply(rope, positions[s], rows, heads * g, d[s], row, d[s], row),
                         lambda: B.ecco_paged8_append(cache, rope, positions[s], at + heads * g * 256, at + heads * (g + 1) * 256, row, slots[s], rows),
                         lambda: B.ecco_paged8_attn(cache, batches[s], g, d[s], row, 128**-0.5, B.ATTN_CAUSAL, outs[s], None, ws, need)):
                call()
                if wait:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        assert B.ecco_kernel_launch_count() == before + 5 * steps              # of the attention's three: the schedule, many rows, few rows
        assert B.ecco_device_status() == 0
        return [*codes, *scales, *outs]

    one_at_a_time = serve(True)
    assert bool((one_at_a_time[2].int() - one_at_a_time[2].int().amin() > 8).any()) and all(bool(o.isfinite().all()) for o in one_at_a_time[4:])
    for _ in range(5):
        for a, b in zip(serve(False), one_at_a_time):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.gpu
def test_callers_on_several_host_threads(B, dev):
    """Four threads, each with a stream, a cache and a workspace of its own, at once: turned, appended and attended to, few rows, many, both, and many by way
    of tiles; against the same calls alone."""
    import threading

    rng = np.random.default_rng(71)
    batches = [([1] * 5, [300, 40, 700, 90, 1200], 8, 4), ([300, 200], [1500, 900], 4, 8), ([1, 2, 300, 1], [500, 800, 3000, 60], 8, 4), ([600, 3], [2000, 700], 2, 8)]
    work = []
    for i, (new, kv, heads, g) in enumerate(batches):
        c = Case(B, rng, new, kv, heads, g, (16, 64, 8, 32)[i], padding=0)
        slots = [int(c.tables[r, t // c.page]) * c.page + t % c.page for r, (a, n) in enumerate(zip(new, kv)) for t in range(n - a, n)]
        tokens = np.concatenate([np.arange(n - a, n) for a, n in zip(new, kv)])
        gen = torch.Generator(device="cuda").manual_seed(72 + i)
        rows = [torch.randn((c.tokens, heads, 128), generator=gen, device="cuda").half() for _ in range(2)]
        rope = B.ecco_rope_init((128, 64, 96, 16)[i], 10000.0 ** (-np.arange((64, 32, 48, 8)[i]) / 64), flags=i & 1)
        work.append(dict(c=c, slots=ints(slots), positions=ints(tokens), rows=rows, rope=rope, ws=torch.empty(c.need(), dtype=torch.uint8, device="cuda"),
                         pools=[p.clone() for p in c.pools], q=torch.empty_like(c.q), out=torch.empty_like(c.q), lse=torch.empty(c.q.shape[:2], device="cuda")))

    def step(w):
        c = w["c"]
        row = c.heads * c.g * 128
        for p, was in zip(c.pools, w["pools"]):
            p.copy_(was)
        w["out"].fill_(7.0)
        B.ecco_rope_apply(w["rope"], w["positions"], c.tokens, c.heads * c.g, c.q, row, w["q"], row)
        B.ecco_paged8_append(c.cache, w["rope"], w["positions"], w["rows"][0], w["rows"][1], c.heads * 128, w["slots"], c.tokens)
        B.ecco_paged8_attn(c.cache, c.batch, c.g, w["q"], row, 128**-0.5, B.ATTN_CAUSAL, w["out"], w["lse"], w["ws"], len(w["ws"]))
        return [t.clone().view(torch.uint8) for t in (*c.pools, w["out"], w["lse"])]

    want = []
    for w in work:
        want.append(step(w))
        torch.cuda.synchronize()
        w["c"].check(w["out"], w["lse"], q=w["q"])
    errors, gate = [], threading.Barrier(len(work))

    def caller(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(10):
                    gate.wait(60)
                    got = [step(work[i]) for _ in range(3)]
                    stream.synchronize()
                    for g in got:
                        for a, b in zip(g, want[i]):
                            assert torch.equal(a, b), batches[i]
        except BaseException as e:                         # told by the main thread
            errors.append(e)
            gate.abort()

    torch.cuda.synchronize()
    threads = [threading.Thread(target=caller, args=(i,)) for i in range(len(work))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    assert B.ecco_device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("new,kv", [([1, 2], [100, 33]), ([4, 1, 3], [700, 40, 5]), ([600], [1500])])
@pytest.mark.parametrize("scale", [2e38, -2e38])
def test_scores_of_zero_under_the_largest_scale(B, dev, new, kv, scale):
    """A row of q of zeros has scores of zero whatever the scale and the blocks' powers of two, of which the products leave fp32: all tokens alike."""
    c = Case(B, np.random.default_rng(new), new, kv, 8, 4, 16, qscale=0.0, exps=(5, 7))
    out, lse = c.run(scale=scale)
    c.check(out, lse, scale=scale)
