// ecco_rope_kernels.cuh -- rotary positions
// Part of the one translation unit ecco_kernels.cu; included from there only.
#pragma once

namespace {

// ---------------------------------------------------------------------------------------------
// Eight lanes to a head, sixteen values each in two 16-byte pieces: pairs 8 s .. 8 s + 7 in lane s, whichever way pairs lie; lanes behind
// the last pair hold what is not turned.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ bool rope_turns(const ecco_rope& r, int s) { return s * 16 < r.rot_dim; }
// the first and the second 16-byte piece of lane s
__device__ __forceinline__ int2 rope_pieces(const ecco_rope& r, int s)
{
    return rope_turns(r, s) && !(r.flags & ECCO_ROPE_NEIGHBOURS) ? make_int2(s, s + r.rot_dim / 16) : make_int2(2 * s, 2 * s + 1);
}
// cos and sin of a pair at a position, times the gain.  The angle is position * turn mod 2^64, in 2^-64 turns, and exact.  What is left of it beside the nearest
// quarter turn, y, is at most pi / 4; the Taylor series to y^9 and y^10 are off by 2e-9 there, roundings included by 2^-23.
__device__ __forceinline__ float2 rope_angle(const ecco_rope& r, int pair, int32_t position)
{
    const uint64_t phase = static_cast<uint64_t>(static_cast<int64_t>(position)) * r.turn[pair];
    const uint32_t quarters = static_cast<uint32_t>(((phase >> 61) + 1) >> 1);                      // to the nearest, mod 4
    const int32_t rest = static_cast<int32_t>(static_cast<int64_t>(phase - (static_cast<uint64_t>(quarters) << 62)) >> 30);        // in 2^-34 turns
    const float y = static_cast<float>(rest) * 3.6572951981e-10f, z = y * y;                        // 2 pi / 2^34
    float s = fmaf(z, 2.7557319224e-6f, -1.9841269841e-4f);
    s = fmaf(s, z, 8.3333333333e-3f);
    s = fmaf(s, z, -1.6666666667e-1f);
    s = fmaf(s * z, y, y);
    float c = fmaf(z, -2.7557319224e-7f, 2.4801587302e-5f);
    c = fmaf(c, z, -1.3888888889e-3f);
    c = fmaf(c, z, 4.1666666667e-2f);
    c = fmaf(c, z, -0.5f);
    c = fmaf(c, z, 1.0f);
    const float a = quarters & 1u ? -s : c, b = quarters & 1u ? c : s;
    const float g = quarters & 2u ? -r.gain : r.gain;
    return make_float2(a * g, r.flags & ECCO_ROPE_INVERSE ? -b * g : b * g);
}
// cos and sin of two pairs, as two fp32 numbers each
struct RopePairs { uint64_t c, s; };
// a lane's sixteen values by its pairs' cos and sin, two pairs at a time
__device__ __forceinline__ void rope_turn(uint4& first, uint4& second, const RopePairs (&cs)[4], bool neighbours)
{
    uint32_t v[8] = {first.x, first.y, first.z, first.w, second.x, second.y, second.z, second.w};
    auto wide = [](uint32_t h) {
        const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&h));
        return pack_f2(x.x, x.y);
    };
    auto narrow = [](uint64_t x) {
        float a, b;
        unpack_f2(x, a, b);
        return pack_h2(a, b);
    };
    auto turned = [&](uint32_t& ah, uint32_t& bh, const RopePairs& k) {
        const uint64_t a = wide(ah), b = wide(bh);
        ah = narrow(fma_f2(b, k.s ^ 0x8000000080000000ull, mul_f2(a, k.c)));
        bh = narrow(fma_f2(b, k.c, mul_f2(a, k.s)));
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (neighbours) {
            uint32_t a = prmt(v[2 * i], v[2 * i + 1], 0x5410u), b = prmt(v[2 * i], v[2 * i + 1], 0x7632u);
            turned(a, b, cs[i]);
            v[2 * i] = prmt(a, b, 0x5410u);
            v[2 * i + 1] = prmt(a, b, 0x7632u);
        } else {
            turned(v[i], v[i + 4], cs[i]);
        }
    }
    first = make_uint4(v[0], v[1], v[2], v[3]);
    second = make_uint4(v[4], v[5], v[6], v[7]);
}
// A row of a table in shared memory: cos of two pairs, then their sin, two pairs of every lane side by side, so that the lanes' loads of 16 bytes
// meet in no bank
struct RopeRow { float v[kGroup]; };
__device__ __forceinline__ void rope_store(RopeRow& row, int pair, float2 cs)
{
    float* const at = row.v + ((pair >> 1 & 3) * 8 + (pair >> 3)) * 4 + (pair & 1);
    at[0] = cs.x;
    at[2] = cs.y;
}
__device__ __forceinline__ void rope_load(RopePairs (&cs)[4], const RopeRow& row, int s)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const ulonglong2 v = reinterpret_cast<const ulonglong2*>(row.v)[i * 8 + s];
        cs[i] = {v.x, v.y};
    }
}

// ---------------------------------------------------------------------------------------------
// K7: rows of heads turned by their positions.  A CTA has eight tokens and a share of their heads: cos and sin are made once and stand in shared
// memory, the first heads on their way meanwhile.  Bound by memory: 512 bytes per token and head (8192 tokens x 40 heads, 168 MB: 28.1 to 28.8 us = 5.8 to 6.0 TB/s, 89 to 91 % of
// the copy rate).
// ---------------------------------------------------------------------------------------------
constexpr int kRopeThreads = 256, kRopeTokens = 8, kRopeInFlight = 4;
constexpr int kRopeTeams = kRopeThreads / 8 / kRopeTokens;             // of eight lanes, to a token

struct RopeRows {
    const int32_t* positions;
    const __half* x;
    __half* out;
    int64_t x_stride, out_stride;
    int32_t n_tokens, n_heads, parts, per_part;            // CTAs to eight tokens, heads to a CTA
};

__global__ void __launch_bounds__(kRopeThreads)
ecco_rope_kernel(const __grid_constant__ ecco_rope rope, const __grid_constant__ RopeRows p)
{
    __shared__ __align__(16) RopeRow table[kRopeTokens];
    const int tid = static_cast<int>(threadIdx.x), s = tid & 7, team = (tid >> 3) % kRopeTeams, local = (tid >> 3) / kRopeTeams;
    const int32_t window = static_cast<int32_t>(blockIdx.x) / p.parts, part = static_cast<int32_t>(blockIdx.x) - window * p.parts;
    const int64_t token0 = static_cast<int64_t>(window) * kRopeTokens, token = token0 + local;
    const int32_t head_end = min(p.n_heads, (part + 1) * p.per_part);
    const int2 piece = rope_pieces(rope, s);
    const bool there = token < p.n_tokens;
    release_dependents();
    dependency_wait();
    uint4 v[kRopeInFlight][2];
    auto load = [&](int32_t head0) {
#pragma unroll
        for (int i = 0; i < kRopeInFlight; ++i) {
            const int32_t head = head0 + i * kRopeTeams;
            if (there && head < head_end) {
                const uint4* const src = reinterpret_cast<const uint4*>(p.x + token * p.x_stride + static_cast<int64_t>(head) * kGroup);
                v[i][0] = __ldcg(src + piece.x);
                v[i][1] = __ldcg(src + piece.y);
            }
        }
    };
    int32_t head0 = part * p.per_part + team;
    load(head0);
    const int pairs = rope.rot_dim / 2;
    for (int i = tid; i < kRopeTokens * (kGroup / 2); i += kRopeThreads) {
        const int t = i / (kGroup / 2), pair = i % (kGroup / 2);
        if (pair < pairs && token0 + t < p.n_tokens) rope_store(table[t], pair, rope_angle(rope, pair, __ldcg(p.positions + token0 + t)));
    }
    __syncthreads();
    if (!there) return;
    const bool turns = rope_turns(rope, s), neighbours = rope.flags & ECCO_ROPE_NEIGHBOURS;
    RopePairs cs[4];
    if (turns) rope_load(cs, table[local], s);
    for (;;) {
#pragma unroll
        for (int i = 0; i < kRopeInFlight; ++i) {
            const int32_t head = head0 + i * kRopeTeams;
            if (head >= head_end) return;
            if (turns) rope_turn(v[i][0], v[i][1], cs, neighbours);
            uint4* const dst = reinterpret_cast<uint4*>(p.out + token * p.out_stride + static_cast<int64_t>(head) * kGroup);
            dst[piece.x] = v[i][0];
            dst[piece.y] = v[i][1];
        }
        head0 += kRopeInFlight * kRopeTeams;
        load(head0);
    }
}

}  // namespace
