"""Rotary positions: ecco_rope_frequencies, ecco_rope_init, ecco_rope_apply.

Reference: angles from exact fractions or in 64 bits, the rotation in 64 bits.  Tolerance of a turned value, from the kernel's roundings:
  cos and sin: what is left of the angle beside the nearest quarter turn, at most pi / 4, rounded to fp32, and the function's own error of up
  to two units, together at most 3 * 2^-24, the product with the gain 2^-24;
  the product, the multiply-and-add and the sum of their errors: 2^-24 of |a| + |b| each;
  |out - ref| <= 2^-11 |ref| + 2^-25 + 8 * 2^-24 * |gain| (|a| + |b|).
"""
import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest

torch = pytest.importorskip("torch")

PI = Fraction(31415926535897932384626433832795028841971693993751058209749445923, 10**64)


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


# ------------------------------------------------------------------ host calls
def frequencies_reference(rot, base, kind, factor, low, high, trained):
    i = np.arange(rot // 2)
    f = base ** (-2.0 * i / rot)
    if kind == 1:
        return f / factor, 1.0
    if kind == 2:
        return (base * factor ** (rot / (rot - 2))) ** (-2.0 * i / rot), 1.0
    if kind == 3:
        turns = trained * f / (2 * math.pi)
        return np.where(turns <= low, f / factor, np.where(turns >= high, f, f / factor + (f - f / factor) * (turns - low) / (high - low))), 1.0
    if kind == 4:
        pair = lambda n: rot / 2 * math.log(trained / (n * 2 * math.pi)) / math.log(base)  # noqa: E731
        lo, hi = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), rot - 1)
        share = np.clip((i - lo) / max(hi - lo, 0.001), 0, 1)
        return f * (1 - share) + f / factor * share, 0.1 * math.log(factor) + 1
    return f, 1.0


@pytest.mark.parametrize("rot", [16, 64, 128])
@pytest.mark.parametrize("kind,factor,low,high,trained", [(0, 1, 1, 4, 0), (1, 4, 1, 4, 0), (2, 8, 1, 4, 0), (3, 8, 1, 4, 8192), (3, 2.5, 0.5, 32, 100), (4, 16, 1, 32, 4096), (4, 1, 1, 2, 70)])
def test_frequencies(B, rot, kind, factor, low, high, trained):
    for base in (10000.0, 500000.0):
        got, gain = B.ecco_rope_frequencies(rot, base, kind, factor, low, high, trained)
        want, want_gain = frequencies_reference(rot, base, kind, factor, low, high, trained)
        assert np.allclose(got, want, rtol=1e-13, atol=0) and abs(gain - want_gain) <= 2.0**-23 * want_gain


def test_fractions_of_a_turn(B):
    rng = np.random.default_rng(3)
    f = np.concatenate([rng.uniform(-20, 20, 30), 10.0 ** rng.uniform(-9, 0, 30), [0.0, 1.0, 2 * math.pi, -1e-300]])
    rope = B.ecco_rope_init(128, f, gain=-0.5, flags=B.ROPE_NEIGHBOURS | B.ROPE_INVERSE)
    assert (rope.gain, rope.rot_dim, rope.flags) == (-0.5, 128, 3)
    for x, turn in zip(f, rope.turn):
        want = Fraction(float(x)) / (2 * PI) % 1 * 2**64
        off = abs(want - turn)
        # a quotient of up to four turns has 62 bits behind the point; one below a turn is within a unit
        assert min(off, 2**64 - off) <= (4 if abs(x) > 6 else 1), x
    assert list(B.ecco_rope_init(32, np.ones(16)).turn)[16:] == [0] * 48


def test_refusals_without_a_gpu(B):
    L, INV, ALIGN = B.lib(), B.ERR_INVALID_ARG, B.ERR_ALIGNMENT
    f, gain = np.ones(64), ctypes.c_float()

    def frequencies(rot=64, base=1e4, kind=4, factor=2.0, low=1.0, high=4.0, trained=100.0, out=f.ctypes.data, g=ctypes.byref(gain)):
        return L.ecco_rope_frequencies(rot, base, ctypes.byref(B.RopeScaling(kind, factor, low, high, trained)), out, g)

    assert frequencies() == 0 and L.ecco_rope_frequencies(64, 1e4, None, f.ctypes.data, ctypes.byref(gain)) == 0
    for bad in (dict(rot=0), dict(rot=8), dict(rot=24), dict(rot=144), dict(rot=-16), dict(base=1.0), dict(base=math.nan), dict(base=math.inf), dict(kind=-1), dict(kind=5),
                dict(factor=0.5), dict(factor=math.nan), dict(factor=math.inf), dict(low=0.0), dict(low=4.0), dict(high=math.inf), dict(trained=0.0), dict(trained=math.nan),
                dict(out=None), dict(g=None), dict(kind=2, factor=1e300, base=1e300)):
        assert frequencies(**bad) == INV, bad
    f = np.ones(64)
    rope = B.Rope()

    def init(rot=64, freq=f, g=1.0, flags=0, to=ctypes.byref(rope)):
        return L.ecco_rope_init(rot, freq.ctypes.data if freq is not None else None, ctypes.c_float(g), flags, to)

    assert init() == 0
    for bad in (dict(rot=0), dict(rot=40), dict(rot=136), dict(freq=None), dict(g=math.nan), dict(g=math.inf), dict(flags=4), dict(to=None),
                dict(freq=np.where(np.arange(64) == 31, np.inf, 1.0)), dict(freq=np.where(np.arange(64) == 0, np.nan, 1.0))):
        assert init(**bad) == INV, bad
    assert init(rot=64, freq=np.where(np.arange(64) == 32, np.nan, 1.0)) == 0                   # beyond the last pair
    with pytest.raises(ValueError):
        B.ecco_rope_init(64, np.ones(64))

    def apply(r=rope, pos=4096, n=3, heads=2, x=8192, xs=256, out=12288, os=256):
        return L.ecco_rope_apply(ctypes.byref(r) if r is not None else None, pos, n, heads, x, xs, out, os, None)

    if not torch.cuda.is_available():
        GONE = B.ERR_CUDA                                  # all arguments fine: the call goes on to ask for the device
        for fine in (dict(), dict(n=2**31 - 1), dict(heads=65535, xs=65535 * 128, os=65535 * 128), dict(xs=(1 << 38) - 8), dict(out=8192)):
            assert apply(**fine) == GONE, fine
    assert apply(n=0) == 0
    broken = [B.Rope.from_buffer_copy(rope) for _ in range(4)]
    broken[0].rot_dim, broken[1].rot_dim, broken[2].gain, broken[3].flags = 0, 130, math.nan, 8
    for bad in (dict(r=None), dict(n=-1), dict(heads=0), dict(heads=65536, xs=1 << 30, os=1 << 30), dict(pos=None), dict(x=None), dict(out=None), dict(xs=248), dict(os=248), dict(xs=-256),
                dict(xs=1 << 38), dict(os=1 << 38), dict(out=8192, os=512), *(dict(r=r) for r in broken)):
        assert apply(**bad) == INV, bad
    for bad in (dict(pos=4098), dict(x=8200), dict(out=12296), dict(xs=260), dict(os=260)):
        assert apply(**bad) == ALIGN, bad


# ------------------------------------------------------------------ the rotation
def turned(x, positions, f, gain, flags, rot):
    """fp64 [tokens][heads][128], and |a| + |b| of every value's pair."""
    y, size = x.astype(np.float64), np.zeros(x.shape)
    turns = [Fraction(float(v)) / (2 * PI) for v in f]
    angle = np.array([[float(int(p) * t % 1) for t in turns] for p in positions]) * 2 * math.pi
    c, s = gain * np.cos(angle)[:, None], gain * np.sin(angle)[:, None]
    if flags & 2:
        s = -s
    i = np.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if flags & 1 else (i, i + rot // 2)
    xa, xb = x[..., a].astype(np.float64), x[..., b].astype(np.float64)
    y[..., a], y[..., b] = xa * c - xb * s, xb * c + xa * s
    size[..., a] = size[..., b] = np.abs(xa) + np.abs(xb)
    return y, size


def check(got, x, positions, f, gain, flags, rot):
    want, size = turned(x, positions, f, gain, flags, rot)
    assert np.all(np.abs(got.astype(np.float64) - want) <= 2.0**-11 * np.abs(want) + 2.0**-25 + 8 * 2.0**-24 * abs(gain) * size)
    assert np.array_equal(got[..., rot:].view(np.uint16), x[..., rot:].view(np.uint16))


@pytest.mark.gpu
@pytest.mark.parametrize("rot", [16, 48, 64, 112, 128])
@pytest.mark.parametrize("flags", [0, 1, 2, 3])
def test_layouts(B, dev, rot, flags):
    rng = np.random.default_rng([rot, flags])
    for tokens, heads in ((1, 1), (7, 3), (9, 17), (130, 5)):
        x = (rng.standard_normal((tokens, heads, 128)) * 10.0 ** rng.integers(-6, 4, (tokens, heads, 1))).astype(np.float16)
        x[0, 0, :5] = [0.0, -0.0, 65504.0, 2.0**-24, -(2.0**-14)]
        positions = rng.integers(-5, 5000, tokens)
        f = 10000.0 ** (-np.arange(rot // 2) * 2 / rot)
        gain = float(np.float32(rng.choice([1.0, 0.37])))
        rope = B.ecco_rope_init(rot, f, gain, flags)
        d = torch.from_numpy(x).cuda()
        out = torch.empty_like(d)
        B.ecco_rope_apply(rope, torch.tensor(positions, dtype=torch.int32, device="cuda"), tokens, heads, d, heads * 128, out, heads * 128)
        check(out.cpu().numpy(), x, positions, f, gain, flags, rot)
        assert np.array_equal(d.cpu().numpy().view(np.uint16), x.view(np.uint16))


@pytest.mark.gpu
@pytest.mark.parametrize("positions", [[0, 1, -1], [2**31 - 1, -(2**31), 2**30 + 1], [131071, 1048575, 16777217], [-(2**31) + 1, 2**24 + 3, 99999999]])
def test_far_positions(B, dev, positions):
    """Angles of positions beyond fp32's whole numbers, of frequencies that have no short fraction."""
    rng = np.random.default_rng(5)
    f = np.concatenate([rng.uniform(0, 7, 40), 10.0 ** rng.uniform(-8, 0, 24)])
    x = rng.standard_normal((3, 4, 128)).astype(np.float16)
    out = torch.empty((3, 4, 128), dtype=torch.float16, device="cuda")
    B.ecco_rope_apply(B.ecco_rope_init(128, f), torch.tensor(positions, dtype=torch.int32, device="cuda"), 3, 4, torch.from_numpy(x).cuda(), 512, out, 512)
    # a turn's fraction is kept to 2^-62 at these frequencies: 2^-31 of a turn at most at the furthest position, within the tolerance
    check(out.cpu().numpy(), x, positions, f, 1.0, 0, 128)


@pytest.mark.gpu
def test_strides_and_in_place(B, dev):
    rng = np.random.default_rng(6)
    tokens, heads, row = 50, 6, 9 * 128 + 8
    x = rng.standard_normal((tokens, row)).astype(np.float16)
    positions = rng.integers(0, 1 << 20, tokens)
    f = 10000.0 ** (-np.arange(32) / 32)
    rope, pos = B.ecco_rope_init(64, f, flags=B.ROPE_NEIGHBOURS), torch.tensor(positions, dtype=torch.int32, device="cuda")
    for at in (0, 128, 8, 3 * 128):                        # heads from the row's begin, behind others, at an address that no head begins at
        d = torch.from_numpy(x).cuda()
        B.ecco_rope_apply(rope, pos, tokens, heads, d.data_ptr() + 2 * at, row, d.data_ptr() + 2 * at, row)
        got = d.cpu().numpy()
        check(np.ascontiguousarray(got[:, at:at + heads * 128]).reshape(tokens, heads, 128), np.ascontiguousarray(x[:, at:at + heads * 128]).reshape(tokens, heads, 128), positions, f, 1.0, 1, 64)
        got[:, at:at + heads * 128] = x[:, at:at + heads * 128]
        assert np.array_equal(got.view(np.uint16), x.view(np.uint16))          # what is beside them stays
        out = torch.full((tokens + 1, heads * 128 + 16), 7.0, dtype=torch.float16, device="cuda")
        B.ecco_rope_apply(rope, pos, tokens, heads, torch.from_numpy(x).cuda().data_ptr() + 2 * at, row, out, heads * 128 + 16)
        assert torch.equal(out[:tokens, :heads * 128].reshape(-1), d[:, at:at + heads * 128].reshape(-1)) and bool((out[:tokens, heads * 128:] == 7).all()) and bool((out[tokens] == 7).all())


@pytest.mark.gpu
def test_not_finite(B, dev):
    x = np.random.default_rng(7).standard_normal((4, 2, 128)).astype(np.float16)
    x[1, 0, 3], x[2, 1, 70], x[3, 0, 5], x[3, 0, 69] = np.nan, np.inf, np.inf, -np.inf
    pos, f = [3, 100, 7, 1], 100.0 ** (-np.arange(64) / 64)
    out = torch.empty((4, 2, 128), dtype=torch.float16, device="cuda")
    B.ecco_rope_apply(B.ecco_rope_init(128, f), torch.tensor(pos, dtype=torch.int32, device="cuda"), 4, 2, torch.from_numpy(x).cuda(), 256, out, 256)
    got = out.cpu().numpy()
    bad = np.zeros(x.shape, bool)
    for t, h, d in ((1, 0, 3), (2, 1, 6), (3, 0, 5)):
        bad[t, h, [d, d + 64]] = True
    assert np.array_equal(~np.isfinite(got), bad)


@pytest.mark.gpu
@pytest.mark.parametrize("flags", [0, 1])
def test_the_inverse_is_the_gradient(B, dev, flags):
    """d<w, R x> / dx: of the formula (the transposed rotation), and by differences; and R^T R x = x."""
    rng = np.random.default_rng([8, flags])
    tokens, heads, rot = 5, 3, 96
    f, positions = 1000.0 ** (-np.arange(48) / 48), rng.integers(0, 9000, tokens)
    pos = torch.tensor(positions, dtype=torch.int32, device="cuda")
    x, w = (rng.standard_normal((tokens, heads, 128)).astype(np.float16) for _ in range(2))

    def run(v, fl):
        out = torch.empty((tokens, heads, 128), dtype=torch.float16, device="cuda")
        B.ecco_rope_apply(B.ecco_rope_init(rot, f, flags=fl), pos, tokens, heads, torch.from_numpy(v).cuda(), heads * 128, out, heads * 128)
        return out.cpu().numpy()

    grad = run(w, flags | B.ROPE_INVERSE)
    check(grad, w, positions, f, 1.0, flags | 2, rot)
    weight = lambda v: float((w.astype(np.float64) * run(v, flags).astype(np.float64)).sum())  # noqa: E731
    for t, h, d in ((0, 0, 0), (1, 2, 47), (2, 1, 48), (3, 0, 95), (4, 2, 127), (0, 1, 95)):
        up, down = x.copy(), x.copy()
        up[t, h, d], down[t, h, d] = 8.0, -8.0             # the map is linear: a large step costs nothing
        # two outputs change, each off by half a step of values up to 16 (2^-7) in both runs; the gradient's own rounding
        i = d if d >= rot else (d ^ 1 if flags else (d + 48) % 96)
        slack = 2 * 2.0**-7 * (abs(float(w[t, h, d])) + abs(float(w[t, h, i]))) / 16 + 2.0**-10 * 4
        assert abs((weight(up) - weight(down)) / 16 - float(grad[t, h, d])) <= slack, (t, h, d)
    back = run(run(x, flags), flags | B.ROPE_INVERSE).astype(np.float64)
    # the first rounding of both of a pair, turned back, and the second
    assert np.abs(back - x).max() <= 2.0**-11 * 3 * np.abs(x.astype(np.float64)).max()


@pytest.mark.gpu
def test_captured_and_on_another_stream(B, dev):
    rng = np.random.default_rng(9)
    x = torch.from_numpy(rng.standard_normal((33, 40, 128)).astype(np.float16)).cuda()
    f = 10000.0 ** (-np.arange(64) / 64)
    rope, pos, out = B.ecco_rope_init(128, f), torch.zeros(33, dtype=torch.int32, device="cuda"), torch.empty_like(x)
    call = lambda: B.ecco_rope_apply(rope, pos, 33, 40, x, 5120, out, 5120)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    rope.turn[0] = 0                                       # the call has read it
    for first in (0, 70000):
        pos.copy_(torch.arange(first, first + 33, dtype=torch.int32))
        graph.replay()
        check(out.cpu().numpy(), x.cpu().numpy(), np.arange(first, first + 33), f, 1.0, 0, 128)


def long_pi(digits):
    """pi as a fraction, by 16 atan(1/5) - 4 atan(1/239) in whole numbers."""
    one = 10 ** (digits + 10)

    def atan_of_inverse(n):
        total, term, k = 0, one // n, 1
        while term:
            total += term // k if k % 4 == 1 else -(term // k)
            term //= n * n
            k += 2
        return total

    return Fraction(16 * atan_of_inverse(5) - 4 * atan_of_inverse(239), one)


def test_fractions_of_frequencies_of_any_size(B):
    """Frequencies of many turns a position: what is left of a turn is as exact as of others.  (The whole turns of 1e308 have 308 digits.)"""
    pi = long_pi(400)
    assert abs(pi - PI) < Fraction(1, 10**63)
    rng = np.random.default_rng(4)
    f = np.concatenate([10.0 ** rng.uniform(0.8, 308, 50) * rng.choice([-1, 1], 50), [1e4, -1e4, 1e9, 2.0**53 + 2, 2.0**64, 2.0**66, 1e100, 1.7e308, -1.7e308, 6.2831853071795862,
                                                                                     6.2831853071795871, 12.566370614359172, -6.283185307179587, 1e22]])
    for x, turn in zip(f, B.ecco_rope_init(128, f).turn):
        off = abs(Fraction(float(x)) / (2 * pi) % 1 * 2**64 - turn)
        # the angle's sine, cosine and arc, its quotient by 2 pi: within a unit each of at most half a turn's last place, and the rounding to 64 bits
        assert min(off, 2**64 - off) <= 4, x


@pytest.mark.gpu
def test_far_positions_of_many_turns_each(B, dev):
    """Frequencies of up to 10^9 turns a position, at the furthest positions: within the same tolerance."""
    rng = np.random.default_rng(10)
    f = 10.0 ** rng.uniform(1, 10, 64) * rng.choice([-1, 1], 64)
    x = rng.standard_normal((4, 4, 128)).astype(np.float16)
    positions = [2**31 - 1, -(2**31), 2**30 + 1, 1]
    out = torch.empty((4, 4, 128), dtype=torch.float16, device="cuda")
    B.ecco_rope_apply(B.ecco_rope_init(128, f), torch.tensor(positions, dtype=torch.int32, device="cuda"), 4, 4, torch.from_numpy(x).cuda(), 512, out, 512)
    # a turn's fraction is within 4 * 2^-64: 2^-31 of a turn at the furthest position
    check(out.cpu().numpy(), x, positions, f, 1.0, 0, 128)


@pytest.mark.parametrize("base", [1.0 + 2.0**-52, 2.0, 10000.0, 1e300])
@pytest.mark.parametrize("low,high,trained", [(1e-310, 1e-309, 1e300), (1e307, 1e308, 1e-300), (1e-320, 1e308, 1.0), (1.0, 1e308, 1e308), (5e-324, 1e-323, 1.7e308), (1e300, 1e301, 5e-324)])
def test_frequencies_at_the_ends_of_the_range(B, base, low, high, trained):
    """Arguments that are allowed give numbers: between the frequency as it is and the slowed one."""
    for rot in (16, 128):
        f = base ** (-2.0 * np.arange(rot // 2) / rot)
        for kind in (B.ROPE_SCALE_BANDS, B.ROPE_SCALE_RAMP):
            got, gain = B.ecco_rope_frequencies(rot, base, kind, 8.0, low, high, trained)
            assert np.all(got <= f * (1 + 1e-13)) and np.all(got >= f / 8 * (1 - 1e-13)) and math.isfinite(gain), (rot, kind)
            # bands: a pair's turns over the trained length; all of these are far from both borders or between them
            if kind == B.ROPE_SCALE_BANDS and not (low < trained / (2 * math.pi) * f.min() < high):
                slow, fast = trained / (2 * math.pi) * f <= low, trained / (2 * math.pi) * f >= high
                assert np.allclose(got[slow], f[slow] / 8, rtol=1e-13, atol=0) and np.allclose(got[fast], f[fast], rtol=1e-13, atol=0)
            # ramp: every pair makes more turns than `high`, or fewer than `low`
            if kind == B.ROPE_SCALE_RAMP and trained / (2 * math.pi) * f.min() > high and base > 1.5:
                assert np.allclose(got, f, rtol=1e-13, atol=0)
