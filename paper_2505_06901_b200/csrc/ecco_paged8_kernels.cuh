// ecco_paged8_kernels.cuh -- K8: the paged KV cache in 8 bits: new tokens into blocks, attention of few rows
// Part of the one translation unit ecco_kernels.cu; included from there only.
#pragma once

namespace {

// ---------------------------------------------------------------------------------------------
// K8a: new tokens into the cache.  A run is what a call brings for one block: rows one after the other whose slots ascend within
// it.  A CTA has the runs that begin in sixteen rows, and a share of their heads; a warp takes a run of one head, of K or of V, as a whole: eight
// lanes to a token, so that its up to 2048 values stay in registers from the load over the rotation and the largest value to the E4M3 numbers.
// Bound by memory, 768 bytes per token and KV head, and not far behind by the issue slots, half busy: 566 instructions to a run (4096 tokens x 32 heads, 101 MB:
// 19.6 to 20.1 us = 5.0 to 5.1 TB/s, 77 to 79 % of the copy rate).  256 windows on 148 SMs leave 40 of these with one CTA of two.
// ---------------------------------------------------------------------------------------------
constexpr int kP8AppendThreads = 256, kP8AppendWarps = kP8AppendThreads / 32, kP8Rows = 16;
constexpr uint32_t kP8RunBytes = kP8Rows * kGroup * 2;     // a run's rows in shared memory: the next one's are on their way while one is dealt with
constexpr uint32_t kP8AppendTable = 128, kP8AppendRuns = kP8AppendTable + 32 * sizeof(RopeRow), kP8AppendSmemBytes = kP8AppendRuns + kP8AppendWarps * 2 * kP8RunBytes;
struct P8Append {
    const int32_t *positions, *slots;
    const __half *k, *v;
    uint8_t *k_codes, *v_codes, *k_scales, *v_scales;
    int64_t token_stride;
    int32_t n_tokens, n_slots, heads, page_shift;
    int32_t kinds, parts;      // CTAs to a window: one of each kind (K, V) or for both, and as many for a share of the heads
};

template <bool kTurn>
__global__ void __launch_bounds__(kP8AppendThreads, 2)
ecco_paged8_append_kernel(const __grid_constant__ ecco_rope rope, const __grid_constant__ P8Append p, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    constexpr unsigned full = 0xffffffffu;
    RopeRow* const table = reinterpret_cast<RopeRow*>(smem + kP8AppendTable);
    const int tid = static_cast<int>(threadIdx.x), lane = tid & 31, warp = tid >> 5, s = lane & 7, team = lane >> 3;
    const int32_t cta = static_cast<int32_t>(blockIdx.x) / p.kinds, kind = static_cast<int32_t>(blockIdx.x) - cta * p.kinds, window = cta / p.parts, part = cta - window * p.parts;
    const int block_shift = min(4, p.page_shift), places = 1 << block_shift;
    const uint32_t bar = smem_u32(smem) + warp * 16, rows_at = smem_u32(smem) + kP8AppendRuns + warp * 2 * kP8RunBytes;
    if (lane < 2) mbar_init(bar + lane * 8, 1);
    __syncwarp();
    release_dependents();
    dependency_wait();
    // lane l: row 16 window - 1 + l.  Runs begin in lanes 1 .. 16 and are sixteen rows at most.
    const int64_t row = static_cast<int64_t>(window) * kP8Rows - 1 + lane;
    int32_t slot = row >= 0 && row < p.n_tokens ? __ldcg(p.slots + row) : -1;
    if (slot >= p.n_slots) slot = -1;
    const int32_t before = __shfl_up_sync(full, slot, 1);
    const bool valid = slot >= 0, begins = valid && (before < 0 || slot >> block_shift != before >> block_shift || slot <= before);
    const unsigned stops = __ballot_sync(full, begins || !valid), starts = __ballot_sync(full, begins) & 0x1fffeu;
    auto run_end = [&](int l) {
        const unsigned behind = l < 31 ? stops >> (l + 1) : 0u;
        return behind ? l + __ffs(behind) : 32;
    };
    const int n_runs = __popc(starts);
    if (n_runs == 0) return;
    // the warp's work: run by run, of each K and V of all heads; a place in it
    struct Item { unsigned left; int of_run, l0, n; };     // runs from this one on, as bits; the item of the run; its first lane and its rows
    const int per_run = p.kinds == 2 ? p.heads : 2 * p.heads, first_v = p.kinds == 2 ? (kind ? 0 : p.heads) : p.heads, step = p.parts * kP8AppendWarps;
    auto open = [&](Item& it) {
        while (it.left && it.of_run >= per_run) { it.of_run -= per_run; it.left &= it.left - 1u; }
        if (!it.left) return;
        it.l0 = __ffs(it.left) - 1;
        it.n = min(run_end(it.l0) - it.l0, kP8Rows);
    };
    // A whole run comes by one copy of sixteen rows, a shorter one row by row: a copy takes ten instructions to issue, whatever its size.
    const int32_t row0 = window * kP8Rows - 1;
    auto fetch = [&](const Item& it, uint32_t stage) {
        if (!it.left) return;
        const bool is_v = it.of_run >= first_v;
        const int head = it.of_run - (is_v ? first_v : 0);
        const uint32_t to = rows_at + stage * kP8RunBytes, b = bar + stage * 8;
        if (lane == 0) mbar_expect_tx(b, it.n * kGroup * 2);
        __syncwarp();
        if (it.n == kP8Rows) {
            if (lane == 0) tma_load_3d(to, is_v ? &v_map : &k_map, 0, head, row0 + it.l0, b);
        } else if (lane < it.n) {
            bulk_g2s(to + lane * kGroup * 2, (is_v ? p.v : p.k) + (static_cast<int64_t>(row0) + it.l0 + lane) * p.token_stride + static_cast<int64_t>(head) * kGroup, kGroup * 2, b);
        }
    };
    Item now = {starts, part * kP8AppendWarps + warp, 0, 0};
    open(now);
    fetch(now, 0);
    if (kTurn && first_v > 0) {
        const int from = __ffs(starts) - 1, to = run_end(31 - __clz(starts)), pairs = rope.rot_dim / 2;
        for (int i = tid; i < (to - from) * (kGroup / 2); i += kP8AppendThreads) {
            const int l = from + i / (kGroup / 2), pair = i % (kGroup / 2);
            const int64_t r = static_cast<int64_t>(window) * kP8Rows - 1 + l;
            if (pair < pairs && r < p.n_tokens) rope_store(table[l], pair, rope_angle(rope, pair, __ldcg(p.positions + r)));
        }
        __syncthreads();
    }
    const int2 turned_piece = kTurn ? rope_pieces(rope, s) : make_int2(2 * s, 2 * s + 1);
    const bool turns = kTurn && rope_turns(rope, s), neighbours = rope.flags & ECCO_ROPE_NEIGHBOURS;
    for (uint32_t nth = 0; now.left; ++nth) {
        Item next = now;
        next.of_run += step;
        open(next);
        fetch(next, (nth + 1) & 1u);
        const int l0 = now.l0, n = now.n, is_v = now.of_run >= first_v, head = now.of_run - (is_v ? first_v : 0);
        now = next;
        const int32_t slot0 = __shfl_sync(full, slot, l0), page = slot0 >> p.page_shift, base = slot0 & ((1 << p.page_shift) - 1) & ~(places - 1);
        const int64_t of_head = static_cast<int64_t>(page) * p.heads + head;
        uint8_t* const block = (is_v ? p.v_codes : p.k_codes) + ((of_head << p.page_shift) + base) * kGroup;
        uint8_t* const scale = (is_v ? p.v_scales : p.k_scales) + (of_head << (p.page_shift - block_shift)) + (base >> block_shift);
        const int2 piece = is_v ? make_int2(2 * s, 2 * s + 1) : turned_piece;
        const bool anew = (slot0 & (places - 1)) == 0;
        int e = kP8Lowest, e_before = kP8Lowest;
        if (!anew) e_before = p8_exponent(__ldcg(scale));
        const uint32_t stage = nth & 1u;
        if (!warp_wait(bar + stage * 8, (nth >> 1) & 1u)) {                        // what is on its way lands before the CTA leaves
            if (now.left) warp_wait(bar + (stage ^ 1u) * 8, ((nth + 1) >> 1) & 1u);
            return;
        }
        uint4 v[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i][0] = v[i][1] = make_uint4(0u, 0u, 0u, 0u);
            if (4 * i + team < n) {
                const uint32_t from = rows_at + stage * kP8RunBytes + (4 * i + team) * kGroup * 2;
                v[i][0] = lds_v4(from + piece.x * 16);
                v[i][1] = lds_v4(from + piece.y * 16);
            }
        }
        __half2 top = __floats2half2_rn(0.0f, 0.0f);       // largest magnitudes; NaN if there is one
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (4 * i >= n) break;
            if (turns && !is_v && 4 * i + team < n) {
                RopePairs cs[4];
                rope_load(cs, table[l0 + 4 * i + team], s);
                rope_turn(v[i][0], v[i][1], cs, neighbours);
            }
            const uint32_t* const w = reinterpret_cast<const uint32_t*>(v[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) top = __hmax2_nan(top, __habs2(*reinterpret_cast<const __half2*>(&w[j])));
        }
        auto bits_of = [](__half2 v) {
            const uint32_t u = *reinterpret_cast<const uint32_t*>(&v);
            return max(u & 0xffffu, u >> 16);
        };
        uint32_t largest = __reduce_max_sync(full, bits_of(top));
        if (largest > 0x7c00u) {                           // NaN becomes zero
            top = __floats2half2_rn(0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t* const w = reinterpret_cast<uint32_t*>(v[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const __half2 h = *reinterpret_cast<const __half2*>(&w[j]);
                    w[j] &= __heq2_mask(h, h);
                    top = __hmax2(top, __habs2(*reinterpret_cast<const __half2*>(&w[j])));
                }
            }
            largest = __reduce_max_sync(full, bits_of(top));
        }
        // 448 is 1.75 times a power of two: a larger mantissa (above 0x300) needs the next one
        e = min(max(static_cast<int>((largest + 0xffu) >> 10) - 23, kP8Lowest), kP8Highest);
        e = max(e, e_before);
        if (!anew && e > e_before) {                       // what the block has already, under the new power of two
            unsigned mine = 0;                             // places that the call brings
            for (int j = 0; j < n; ++j) mine |= 1u << (__shfl_sync(full, slot, l0 + j) & (places - 1));
            const uint32_t shrink = power_h2(e_before - e);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int place = 4 * i + team;
                if (place >= places || (mine >> place & 1u)) continue;
                uint4* const at = reinterpret_cast<uint4*>(block + place * kGroup) + s;
                uint4 x = __ldcg(at);
                auto again = [&](uint32_t c) { return to_e4m3(mul_h2(e4m3_low(c), shrink), mul_h2(e4m3_high(c), shrink)); };
                *at = make_uint4(again(x.x), again(x.y), again(x.z), again(x.w));
            }
        }
        if (lane == 0) *scale = static_cast<uint8_t>(e + 127);
        const uint32_t inverse = power_h2(-e);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (4 * i >= n) break;
            const int32_t to = __shfl_sync(full, slot, min(l0 + 4 * i + team, 31)) & (places - 1);
            if (4 * i + team >= n) continue;
            auto codes = [&](const uint4& x) {
                return make_uint2(to_e4m3(mul_h2(x.x, inverse), mul_h2(x.y, inverse)), to_e4m3(mul_h2(x.z, inverse), mul_h2(x.w, inverse)));
            };
            const uint2 a = codes(v[i][0]), b = codes(v[i][1]);
            uint8_t* const dst = block + to * kGroup;
            if (piece.y == piece.x + 1) {
                reinterpret_cast<uint4*>(dst)[s] = make_uint4(a.x, a.y, b.x, b.y);
            } else {
                reinterpret_cast<uint2*>(dst)[piece.x] = a;
                reinterpret_cast<uint2*>(dst)[piece.y] = b;
            }
        }
    }
}

// rows of a request that ecco_paged8_few_kernel takes together
constexpr int kP8Rows16 = 16;
__device__ __forceinline__ int32_t p8_row_groups(int64_t rows) { return static_cast<int32_t>((rows + kP8Rows16 - 1) / kP8Rows16); }
// a request's tiles in the line of ecco_paged8_few_kernel: once for each sixteen rows
__device__ __forceinline__ int64_t p8_line_tiles(const PagedReq& q, int32_t q_per_kv, int32_t few_rows)
{
    const int64_t rows = static_cast<int64_t>(q.rows) * q_per_kv;
    return rows > few_rows ? 0 : static_cast<int64_t>(p8_row_groups(rows)) * ((q.kv + 31) >> 5);
}
// The line never passes this, whatever the arrays hold: sums of requests that share no tile do not reach it.
__device__ __forceinline__ int64_t p8_line_limit(int32_t T, int32_t few_rows) { return static_cast<int64_t>(T) * p8_row_groups(few_rows); }
// by one warp: rows of requests whose lanes say so get zeros and -infinity
__device__ __forceinline__ void p8_empty_rows(const PagedKv& kv, const PagedOut& o, const PagedReq& q, bool empty)
{
    constexpr unsigned full = 0xffffffffu;
    const int lane = static_cast<int>(threadIdx.x & 31u);
    for (unsigned left = __ballot_sync(full, empty); left; left &= left - 1u) {
        const int src = __ffs(left) - 1;
        const int64_t row0 = __shfl_sync(full, q.row0, src), n = static_cast<int64_t>(__shfl_sync(full, q.rows, src)) * o.q_heads;
        for (int64_t i = 0; i < n; ++i) {
            const int64_t at = row0 * o.q_heads + i;
            reinterpret_cast<uint2*>(o.out + at * kGroup)[lane] = make_uint2(0u, 0u);
            if (o.lse && lane == 0) o.lse[at] = -INFINITY;
        }
    }
}
// K8s: by the first warp, what the attention kernels need to know of a batch: the blocks of requests of many rows (paged_schedule) and, of more requests than
// ecco_paged8_few_kernel keeps in shared memory, its line.
// with_tiles: the others bring the pages of the requests of many rows into fp16 tiles, which ecco_paged_many_kernel reads as it does those of K6s.  A warp has
// a tile of K and of V: four tokens a load, 32 bytes of a piece a lane and store.
constexpr int kP8StageWarps = 8;
__global__ void __launch_bounds__(kP8StageWarps * 32, 2)
ecco_paged8_stage_kernel(const __grid_constant__ PagedKv kv, const __grid_constant__ PagedOut o, const __grid_constant__ PagedSchedule sc, int32_t with_tiles,
                         int32_t with_line)
{
    constexpr unsigned full = 0xffffffffu;
    __shared__ int32_t firsts[kStageTiles + 1];
    const int lane = static_cast<int>(threadIdx.x & 31u), warp = static_cast<int>(threadIdx.x >> 5), block_shift = min(4, kv.page_shift);
    release_dependents();
    dependency_wait();
    fetch_firsts(kv, firsts);
    const int32_t T = paged_tiles(kv);
    if (blockIdx.x == 0 && warp == 0) {
        if (lane == 0 && __ldcg(kv.kv_tiles + kv.n_req) > kv.max_tiles) atomicExch(&g_device_status, ECCO_ERR_INVALID_ARG);
        paged_schedule(kv, sc, o);
        if (with_line) {                                   // more requests than ecco_paged8_few_kernel keeps in shared memory
            int64_t line = 0;
            const int64_t limit = p8_line_limit(T, sc.few_rows);
            for (int r0 = 0; r0 < kv.n_req; r0 += 32) {
                PagedReq q = {};
                if (r0 + lane < kv.n_req) q = paged_req(kv, r0 + lane, T);
                int64_t upto = p8_line_tiles(q, o.q_per_kv, sc.few_rows);
                p8_empty_rows(kv, o, q, q.rows > 0 && static_cast<int64_t>(q.rows) * o.q_per_kv <= sc.few_rows && q.kv == 0);
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int64_t x = __shfl_up_sync(full, upto, d);
                    if (lane >= d) upto += x;
                }
                upto = min(line + upto, limit);
                if (r0 + lane < kv.n_req) sc.few_tiles[r0 + lane + 1] = static_cast<int32_t>(upto);
                line = __shfl_sync(full, upto, 31);
            }
        }
        return;
    }
    if (!with_tiles) return;                               // there is no room for any
    const int64_t units = static_cast<int64_t>(T) * kv.heads, warps = static_cast<int64_t>(gridDim.x) * kP8StageWarps - 1;
    for (int64_t u = static_cast<int64_t>(blockIdx.x) * kP8StageWarps + warp - 1; u < units; u += warps) {
        const int32_t head = static_cast<int32_t>(divide(static_cast<uint64_t>(u), static_cast<uint64_t>(T))), tile = static_cast<int32_t>(u - static_cast<int64_t>(head) * T);
        int32_t first;
        const int r = request_of(kv, firsts, tile, first);
        const PagedReq q = paged_req(kv, r, T);
        // lane l: where token l is
        const int64_t token = (static_cast<int64_t>(tile) - first) * 32 + lane, entry = token >> kv.page_shift;
        int32_t page = -2;
        if (token >= 0 && entry < kv.stride) page = __ldcg(kv.tables + static_cast<int64_t>(r) * kv.stride + entry);     // whether or not it is needed
        if (static_cast<int64_t>(q.rows) * o.q_per_kv <= sc.few_rows) continue;
        if (token < 0 || token >= q.kv) {
            page = -1;
        } else if (page < 0 || page >= kv.n_pages) {
            atomicExch(&g_device_status, ECCO_ERR_INVALID_ARG);
            page = -1;
        }
        const int64_t of_head = static_cast<int64_t>(max(page, 0)) * kv.all_heads + kv.head0 + head;
        const int32_t place = static_cast<int32_t>(token & ((1 << kv.page_shift) - 1));
        const int64_t at = (of_head << kv.page_shift) + place, of_scale = (of_head << (kv.page_shift - block_shift)) + (place >> block_shift);
        uint32_t scale[2] = {127, 127};
        if (page >= 0) { scale[0] = __ldcg(kv.k_meta + of_scale); scale[1] = __ldcg(kv.v_meta + of_scale); }
        uint4 v[2][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int t = 4 * i + (lane >> 3);
            const int64_t from = __shfl_sync(full, at, t) * kGroup;
            const bool there = __shfl_sync(full, page, t) >= 0;
            v[0][i] = v[1][i] = make_uint4(0u, 0u, 0u, 0u);
            if (there) {
                v[0][i] = __ldcg(reinterpret_cast<const uint4*>(kv.k_blocks + from) + (lane & 7));
                v[1][i] = __ldcg(reinterpret_cast<const uint4*>(kv.v_blocks + from) + (lane & 7));
            }
        }
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const uint32_t by_lane = power_h2(p8_exponent(scale[which]));
            uint8_t* const dst = staged_tile(kv, which, head, tile) + (lane & 7) * kPieceBytes;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int t = 4 * i + (lane >> 3);
                const uint32_t by = __shfl_sync(full, by_lane, t);
                const uint32_t c[4] = {v[which][i].x, v[which][i].y, v[which][i].z, v[which][i].w};
                uint32_t h[8];
#pragma unroll
                for (int j = 0; j < 4; ++j) { h[2 * j] = mul_h2(e4m3_low(c[j]), by); h[2 * j + 1] = mul_h2(e4m3_high(c[j]), by); }
                const bool swapped = (t >> 2) & 1;
                const uint32_t out[8] = {swapped ? h[4] : h[0], swapped ? h[5] : h[1], swapped ? h[6] : h[2], swapped ? h[7] : h[3],
                                         swapped ? h[0] : h[4], swapped ? h[1] : h[5], swapped ? h[2] : h[6], swapped ? h[3] : h[7]};
                stg_v8(dst + t * 32, out);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------
// K8f: attention of requests of few rows (new tokens x query heads per KV head), straight from the pages.
// All tiles of 32 tokens of all requests and heads, once for each sixteen rows, form one line, cut into equal parts for the CTAs and, in these, for eight
// warps.  Four more warps bring a warp's tiles from the pages into its ring in shared memory.  A warp takes a tile into registers and does
//   S^T = K Q^T   tokens x rows, mma.sync: a lane's four consecutive E4M3 numbers are its part of a step of sixteen dims, Q having the same order
//   the softmax   in fp32; K's power of two is a factor of the score, V's goes into the weight: w = 2^(s + e - m), sum of 2^-e w
//   O^T = V^T W   two tokens' bytes side by side become the fp16 pair that an operand wants, W turned by movmatrix
// so that the conversion from E4M3 is all that lies between shared memory and the tensor cores.
// Pieces of a request that lie in several warps of a CTA are joined in shared memory, those in several CTAs by the CTA that comes last, in their order: the
// result does not depend on who that is.
// Bound by memory, 256 bytes per token and KV head, where there is much of it: 32 requests of up to 16384 tokens, 8 heads of 8 rows, 589 MB: 104 to 109 us = 5.4 to 5.7 TB/s,
// 82 to 86 % of the copy rate; all but some 10 us of them at 6.2.  A tile takes a warp some 1250 clocks without its loads, 340 of an SM's are what memory allows.  Else by the way
// through one tile: launch, lengths, pages, a tile from memory, its products, and the join, some 9 us.
// ---------------------------------------------------------------------------------------------
constexpr int kP8Warps = 8, kP8Loaders = 4, kP8Threads = (kP8Warps + kP8Loaders) * 32, kP8Stages = 2, kP8Reqs = 512;
constexpr uint32_t kP8TileBytes = 32 * kGroup;             // of K or of V
constexpr uint32_t kP8StageBytes = 2 * kP8TileBytes, kP8ScaleBytes = 32 * 16;          // beside it words that the blocks' powers of two are in, and where in these
struct alignas(16) P8Piece { int64_t begin; int32_t units, head, row0, rows, group, valid; };
struct P8Span { int64_t begin; int32_t units, head, row0, rows, group, valid, lo, hi; };
// Shared memory of a kernel for kN times eight rows.
template <int kN> struct P8Smem {
    static constexpr int kWarps = kP8Warps;
    static constexpr uint32_t kPieceBytes = kN * 8 * kGroup * 4;                  // sums of a piece
    // barriers: a warp's tiles have come, are free again
    static constexpr uint32_t kFree = kWarps * kP8Stages * 8, kPieces = 2 * kFree, kSpans = kPieces + kWarps * 2 * sizeof(P8Piece), kMl = kSpans + 128;
    static constexpr uint32_t kLists = kMl + kWarps * 2 * kN * 8 * 8, kListBytes = 4 * (kP8Reqs + 4) * 4;          // the line, lengths, first rows and rows of the requests
    static constexpr uint32_t kScales = (kLists + kListBytes + 15) / 16 * 16, kFirst = kScales + kWarps * kP8Stages * kP8ScaleBytes;
    static constexpr uint32_t kRing = (kFirst + kWarps * kPieceBytes + 1023) / 1024 * 1024, kBytes = kRing + kWarps * kP8Stages * kP8StageBytes;
    static_assert(2 * sizeof(P8Span) <= 112 && kPieces % 16 == 0 && kLists % 16 == 0 && kBytes <= kSmemCtaBytes && kP8Stages * kP8StageBytes >= kPieceBytes, "fits an SM");
};

struct P8Few {
    const int32_t* line;       // [n_req + 1], or NULL: the kernel makes it
    int32_t few_rows, by_request;
    float* part;               // [CTA][first, last][kP8Rows16][128]
    float2* part_ml;           // [CTA][first, last][kP8Rows16]
    Ticket* tickets;           // [CTA * kTicketStride]
    Ticket tag;
};
// as mma_16816, for the compiler to place
__device__ __forceinline__ void mma_h2(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t turn_8x8(uint32_t v)
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

// kN: eight rows each, of a piece
template <int kN>
__global__ void __launch_bounds__(kP8Threads, 1)
ecco_paged8_few_kernel(const __grid_constant__ PagedKv kv, const __grid_constant__ PagedOut o, const __grid_constant__ P8Few f, const __grid_constant__ CUtensorMap k_map,
                       const __grid_constant__ CUtensorMap v_map)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    using Smem = P8Smem<kN>;
    constexpr int kRows = kN * 8;
    constexpr unsigned full = 0xffffffffu;
    const int tid = static_cast<int>(threadIdx.x);
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3u, base = smem_u32(smem);
    int32_t* const line = reinterpret_cast<int32_t*>(smem + Smem::kLists);
    int32_t *const kvs = line + kP8Reqs + 4, *const row0s = kvs + kP8Reqs + 4, *const rows_of = row0s + kP8Reqs + 4;
    P8Piece* const pieces = reinterpret_cast<P8Piece*>(smem + Smem::kPieces);              // [warp][first, last]
    P8Span* const spans = reinterpret_cast<P8Span*>(smem + Smem::kSpans);
    volatile int* const joins = reinterpret_cast<volatile int*>(smem + Smem::kSpans + 112);
    float2* const ml = reinterpret_cast<float2*>(smem + Smem::kMl);                        // [warp][first, last][row]
    int64_t* const sums = reinterpret_cast<int64_t*>(smem + Smem::kFirst);                 // before there are pieces
    const int piece_shift = min(5, kv.page_shift), block_shift = min(4, kv.page_shift), n_blocks = 32 >> block_shift;      // of a tile
    if (tid < kP8Warps * kP8Stages) {
        mbar_init(base + tid * 8, 2 * min(n_blocks, 16));
        mbar_init(base + Smem::kFree + tid * 8, 1);
    }
    if (tid < kP8Warps * 2) pieces[tid].valid = 0;
    __syncthreads();
    // Behind ecco_paged_many_kernel the wait comes at the end, on the conditions that stand at ecco_paged_few_kernel: what is read here was there before
    // that kernel began, it is read through L2 alone (the tensor maps' and bulk copies, __ldcg; the powers of two by __ldcg, too, and not by copy_word), and
    // neither writes what the other reads or writes.
    if (!o.early) dependency_wait();
    release_dependents();
    const int32_t T = paged_tiles(kv);
    if (!f.line) {
        // the line: prefix sums over the requests, in rounds of a request per thread.  Mostly it is kv_tiles as it stands: no request that would
        // be in the line twice, or not at all, or whose lengths say something else.
        if (tid == 0) {
            line[0] = 0;
            if (blockIdx.x == 0 && __ldcg(kv.kv_tiles + kv.n_req) > kv.max_tiles) atomicExch(&g_device_status, ECCO_ERR_INVALID_ARG);
        }
        auto keep = [&](int r, const PagedReq& q, int32_t upto) {
            line[r + 1] = upto;
            kvs[r] = q.kv;
            row0s[r] = q.row0;
            rows_of[r] = q.rows;
        };
        PagedReq q = {};
        bool plain = kv.n_req <= kP8Threads;
        if (plain && tid < kv.n_req) {
            q = paged_req(kv, tid, T);
            plain = !q.cut && q.rows > 0 && q.rows <= kv.max_new && q.rows * o.q_per_kv <= kP8Rows16 && q.kv > 0 && q.tiles == (q.kv + 31) >> 5 && (tid > 0 || q.first == 0);
            keep(tid, q, q.first + q.tiles);
        }
        if (!__syncthreads_and(plain)) {
            int64_t before = 0;
            const int64_t limit = p8_line_limit(T, f.few_rows);
            for (int r0 = 0; r0 < kv.n_req; r0 += kP8Threads) {
                const int r = r0 + tid;
                if (kv.n_req > kP8Threads) {               // else it is at hand
                    q = {};
                    if (r < kv.n_req) q = paged_req(kv, r, T);
                }
                if ((q.cut || q.rows > kv.max_new) && blockIdx.x == 0) atomicExch(&g_device_status, ECCO_ERR_INVALID_ARG);
                int64_t upto = p8_line_tiles(q, o.q_per_kv, f.few_rows);
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int64_t x = __shfl_up_sync(full, upto, d);
                    if (static_cast<int>(lane) >= d) upto += x;
                }
                if (lane == 31) sums[warp] = upto;
                __syncthreads();
                int64_t all = 0;
#pragma unroll
                for (int w = 0; w < kP8Threads / 32; ++w) {
                    if (w < static_cast<int>(warp)) upto += sums[w];
                    all += sums[w];
                }
                if (r < kv.n_req) keep(r, q, static_cast<int32_t>(min(before + upto, limit)));
                before = min(before + all, limit);
                // requests without a token: nobody else comes to their rows
                if (r0 / kP8Threads % static_cast<int>(gridDim.x) == static_cast<int>(blockIdx.x))
                    p8_empty_rows(kv, o, q, q.rows > 0 && static_cast<int64_t>(q.rows) * o.q_per_kv <= f.few_rows && q.kv == 0);
                __syncthreads();
            }
        }
    }
    auto line_at = [&](int r) { return f.line ? __ldcg(f.line + r) : line[r]; };
    const int32_t L = line_at(kv.n_req);
    const int64_t U = static_cast<int64_t>(L) * kv.heads;
    const UnitSplit cta_split(U, static_cast<int>(gridDim.x));
    int64_t c0 = cta_split.begin(static_cast<int>(blockIdx.x)), c1 = cta_split.begin(static_cast<int>(blockIdx.x) + 1);
    if (f.by_request) {                                    // a CTA to a request and head
        const int32_t head = static_cast<int32_t>(blockIdx.x) / kv.n_req, r = static_cast<int32_t>(blockIdx.x) - head * kv.n_req;
        c0 = static_cast<int64_t>(head) * L + line_at(r);
        c1 = static_cast<int64_t>(head) * L + line_at(r + 1);
    }
    const UnitSplit split(c1 - c0, kP8Warps);

    // a place in the line: unit u is tile `tile` of a piece, i.e. of sixteen rows (group) of a request for a head, which has units [begin, begin + units)
    struct Place { int64_t u, begin, end; int32_t units, head, tile, r, kv, row0, rows, group; };
    // the piece that unit p.u is of, of request p.r or one behind it (r = 0: any); end: at most `stop`.  Every lane for itself.
    auto seek = [&](Place& p, int64_t stop) {
        if (p.u >= stop) return;
        const int32_t nth = static_cast<int32_t>(divide(static_cast<uint64_t>(p.u), static_cast<uint64_t>(L))), off = static_cast<int32_t>(p.u - static_cast<int64_t>(nth) * L);
        int r = nth == p.head ? p.r : 0;
        int32_t to = line_at(r + 1);
        for (int i = 0; i < 2 && to <= off; ++i) to = line_at(++r + 1);
        if (to <= off) {
            for (int n = kv.n_req - r; n > 1;) {           // the last request that begins at or before the place
                const int half = n >> 1;
                if (line_at(r + half) <= off) { r += half; n -= half; } else n = half;
            }
            to = line_at(r + 1);
        }
        const int32_t from = line_at(r);
        if (f.line) {
            const PagedReq q = paged_req(kv, r, T);
            p.kv = q.kv; p.row0 = q.row0; p.rows = q.rows;
        } else {
            p.kv = kvs[r]; p.row0 = row0s[r]; p.rows = rows_of[r];
        }
        const int32_t tiles = max((p.kv + 31) >> 5, 1);
        p.r = r;
        p.head = nth;
        p.group = off - from < tiles ? 0 : (off - from) / tiles;
        const int32_t at = from + p.group * tiles;
        p.begin = static_cast<int64_t>(nth) * L + at;
        p.units = min(tiles, to - at);
        p.end = min(p.begin + p.units, stop);
        p.tile = off - at;
    };
    const int32_t in_page = (1 << kv.page_shift) - 1;
    if (warp >= kP8Warps) {
        // Loads: half a warp to a warp's ring, a lane to a block or two of a tile.  A tile's pages are looked up with the tile before it; nothing else from memory
        // passes through registers on its way, but for the powers of two behind ecco_paged_many_kernel.  384 threads x 168 registers = 128 x 72 + 256 x 216.  (Each warp with its own loads, half of a tile's 2400 clocks
        // went into these; one warp with all of them came too late: 8 requests of 4050 tokens, 32 heads 59 and 62 us.)
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        const int w = static_cast<int>(warp - kP8Warps) * 2 + static_cast<int>(lane >> 4), j = static_cast<int>(lane & 15u);
        const uint32_t full_at = base + w * kP8Stages * 8, free_at = full_at + Smem::kFree, ring = base + Smem::kRing + w * kP8Stages * kP8StageBytes;
        const uint32_t scales = base + Smem::kScales + w * kP8Stages * kP8ScaleBytes;
        const int64_t n_scales = static_cast<int64_t>(kv.n_pages) * kv.all_heads << (kv.page_shift - block_shift);
        const int64_t stop = j < n_blocks ? c0 + split.begin(w + 1) : 0;
        Place p = {};
        p.u = j < n_blocks ? c0 + split.begin(w) : 0;
        seek(p, stop);
        // the page of a block of the tile that p is at: -1: none, -2: there is nothing to look for
        auto page_of = [&](int i) {
            const int32_t token = p.tile * 32 + (i << block_shift), e = token >> kv.page_shift;
            if (p.u >= stop || token >= p.kv) return -2;
            return e < kv.stride ? max(__ldcg(kv.tables + static_cast<int64_t>(p.r) * kv.stride + e), -1) : -1;
        };
        int32_t page_next = page_of(j);
        uint32_t n = 0;
        int idle = 0;
        while (__any_sync(full, p.u < stop)) {
            const uint32_t stage = n % kP8Stages;
            const bool go = p.u < stop && (n < kP8Stages || mbar_test(free_at + stage * 8, (n / kP8Stages - 1) & 1u));
            if (go) {
                const uint32_t b = full_at + stage * 8;
                auto ask = [&](int i, int32_t page) {
                    const uint32_t words = scales + stage * kP8ScaleBytes + i * 16;
                    if (page == -1 || page >= kv.n_pages) atomicExch(&g_device_status, ECCO_ERR_INVALID_ARG);
                    if (page < 0 || page >= kv.n_pages) {  // nobody sees the block, or what is seen is unspecified
                        sts_v4(words, 127u, 127u, 0u, 0u);
                        return;
                    }
                    const int32_t head = kv.head0 + p.head, place = (p.tile * 32 + (i << block_shift)) & in_page;
                    const int64_t of_head = static_cast<int64_t>(page) * kv.all_heads + head;
                    if (((i << block_shift) & ((1 << piece_shift) - 1)) == 0) {
                        const uint32_t to = ring + stage * kP8StageBytes + (i << (block_shift + 7)), bytes = 1u << (piece_shift + 7);
                        mbar_expect_more(b, 2 * bytes);
                        if (kv.page_shift >= kP8SwizzledShift) {
                            tma_load_4d(to, &k_map, 0, place, head, page, b);
                            tma_load_4d(to + kP8TileBytes, &v_map, 0, place, head, page, b);
                        } else {
                            const int64_t from = ((of_head << kv.page_shift) + place) * kGroup;
                            bulk_g2s(to, kv.k_blocks + from, bytes, b);
                            bulk_g2s(to + kP8TileBytes, kv.v_blocks + from, bytes, b);
                        }
                    }
                    const int64_t scale = (of_head << (kv.page_shift - block_shift)) + (place >> block_shift), word = scale & ~3ll;
                    if (o.early) {                         // through L2: copy_word goes through L1, where older bytes may be before the wait
                        sts_v4(words, __ldcg(kv.k_meta + scale), __ldcg(kv.v_meta + scale), 0u, 0u);
                        return;
                    }
                    const int there = static_cast<int>(min(n_scales - word, static_cast<int64_t>(4)));
                    copy_word(words, kv.k_meta + word, there);
                    copy_word(words + 4, kv.v_meta + word, there);
                    sts_u32(words + 8, static_cast<uint32_t>(scale & 3) * 8);
                };
                ask(j, page_next);
                if (j + 16 < n_blocks) ask(j + 16, page_of(j + 16));   // pages of one token
                arrive_with_words(b);
                mbar_arrive(b);                            // and with what has been written here
                ++n;
                ++p.tile;
                if (++p.u == p.end) seek(p, stop);
                page_next = page_of(j);
            }
            idle = __any_sync(full, go) ? 0 : idle + 1;
            if (idle > kWaitLimit) {                       // a warp has given up: what is on its way lands before the CTA leaves
                if (lane == 0) atomicExch(&g_device_status, ECCO_ERR_DEVICE_TIMEOUT);
                for (uint32_t i = n < kP8Stages ? 0 : n - kP8Stages; i < n; ++i)
                    for (int k = 0; k < kWaitLimit && !mbar_test(full_at + (i % kP8Stages) * 8, (i / kP8Stages) & 1u); ++k) {}
                break;
            }
        }
        return;
    }
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    auto meet = [&]() { asm volatile("bar.sync 1, %0;" ::"n"(kP8Warps * 32) : "memory"); };          // the warps with tiles, without those that load them
    const uint32_t bar = base + warp * kP8Stages * 8, ring = base + Smem::kRing + warp * kP8Stages * kP8StageBytes;
    const uint32_t scales = base + Smem::kScales + warp * kP8Stages * kP8ScaleBytes, swizzle = kv.page_shift >= kP8SwizzledShift ? 7u : 0u;
    const int64_t u0 = c0 + split.begin(static_cast<int>(warp)), u1 = c0 + split.begin(static_cast<int>(warp) + 1);
    Place at = {};
    at.u = u0;
    seek(at, u1);
    uint32_t taken = 0;
    // pieces of this CTA that other CTAs have parts of: at its begin and at its end
    if (!f.by_request && warp == kP8Warps - 1) {
        Place p = {};
        P8Span sp[2] = {};
        for (int i = 0; i < 2; ++i) {
            p.u = i ? c1 - 1 : c0;
            if (c0 < c1) seek(p, c1);
            const bool out = c0 < c1 && (p.begin < c0 || p.begin + p.units > c1) && !(i && sp[0].valid && sp[0].begin == p.begin);
            sp[i] = P8Span{p.begin, p.units, p.head, p.row0, p.rows, p.group, out, 0, 0};
            if (out) {
                sp[i].lo = cta_split.owner(p.begin);
                sp[i].hi = cta_split.owner(p.begin + p.units - 1);
                if (lane == 0) {
                    Ticket* const word = f.tickets + static_cast<int64_t>(sp[i].lo) * kTicketStride;
                    claim_ticket(word, look_at_ticket(word), f.tag);
                }
            }
            if (lane == 0) spans[i] = sp[i];
        }
    }

    bool ok = true;
    while (ok && at.u < u1) {
        const int R = min(at.rows * o.q_per_kv - at.group * kP8Rows16, kN * 8);
        const int64_t from_u = at.u;
        // Q: lane (row g, c) has dims 32 c .. 32 c + 31, which are its part of all steps; what belongs to no row is zero
        uint32_t q[kN][16];
        int32_t seen[kN][2];
#pragma unroll
        for (int n = 0; n < kN; ++n) {
            const int row = n * 8 + static_cast<int>(g), i = at.group * kP8Rows16 + row, token = i / o.q_per_kv, h = i - token * o.q_per_kv;
            const uint4* const src = reinterpret_cast<const uint4*>(o.q + static_cast<int64_t>(at.row0 + token) * o.q_stride + (static_cast<int64_t>(kv.head0 + at.head) * o.q_per_kv + h) * kGroup) + c * 4;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint4 v = row < R ? __ldcg(src + j) : make_uint4(0u, 0u, 0u, 0u);
                q[n][4 * j] = v.x; q[n][4 * j + 1] = v.y; q[n][4 * j + 2] = v.z; q[n][4 * j + 3] = v.w;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int mine = n * 8 + static_cast<int>(c) * 2 + e;
                seen[n][e] = mine < R ? tokens_seen(PagedReq{0, 0, at.kv, at.row0, at.rows, false}, (at.group * kP8Rows16 + mine) / o.q_per_kv, o.causal) : at.kv;
            }
        }
        int32_t least = at.kv;                             // that a row sees (rows that there are not, with zeros for q, see all)
#pragma unroll
        for (int n = 0; n < kN; ++n) least = min(least, min(seen[n][0], seen[n][1]));
        const int32_t tile_of_masks = __reduce_min_sync(full, least) >> 5;
        float acc[8][kN][4], m[kN][2], l[kN][2];
#pragma unroll
        for (int n = 0; n < kN; ++n) {
#pragma unroll
            for (int e = 0; e < 2; ++e) { m[n][e] = -INFINITY; l[n][e] = 0.0f; }
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[j][n][e] = 0.0f;
        }
        for (; at.u < at.end; ++at.u, ++at.tile) {
            const uint32_t stage = taken % kP8Stages, k_at = ring + stage * kP8StageBytes, v_at = k_at + kP8TileBytes, s_at = scales + stage * kP8ScaleBytes;
            ok = warp_wait(bar + stage * 8, (taken / kP8Stages) & 1u);
            if (!ok) break;
            ++taken;
            // The tile goes into registers, K as the scores need it: token mt * 16 + g and the eighth behind it, dims 32 c .. 32 c + 31; V as the second
            // products need it: tokens 2 c, 2 c + 1, 2 c + 8, 2 c + 9 of sixteen, dims 16 g .. 16 g + 15.  With eight rows both find room at once, and the
            // place in the ring is free again before there is any product.
            uint4 kx[2][2][2], vx[2][4];
            auto load_v = [&]() {
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) vx[kt][i] = lds_v4(v_at + (kt * 16 + 2 * c + (i & 1) + (i >> 1) * 8) * kGroup + (g ^ ((2 * c + (i & 1)) & swizzle)) * 16);
            };
            uint4 words[2][2];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    words[mt][h] = h == 0 || block_shift < 4 ? lds_v4(s_at + ((mt * 16 + h * 8 + g) >> block_shift) * 16) : words[mt][0];
#pragma unroll
                    for (int half = 0; half < 2; ++half) kx[mt][h][half] = lds_v4(k_at + (mt * 16 + h * 8 + g) * kGroup + ((2 * c + half) ^ (g & swizzle)) * 16);
                }
            if (kN == 1) {
                load_v();
                warp_arrive(bar + Smem::kFree + stage * 8);            // the whole warp has read the tile
            }
            float4 by[2][2];                               // K's power of two, V's exponent, the inverse of V's power of two
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (h && block_shift == 4) {
                        by[mt][h] = by[mt][0];
                        continue;
                    }
                    const uint4 x = words[mt][h];
                    const int k = p8_exponent((x.x >> x.z) & 0xffu), v = p8_exponent((x.y >> x.z) & 0xffu);
                    by[mt][h] = make_float4(__uint_as_float(static_cast<uint32_t>(k + 127) << 23), static_cast<float>(v), __uint_as_float(static_cast<uint32_t>(127 - v) << 23), 0.0f);
                }
            // scores: sixteen tokens x eight rows; with eight rows in two sums each, for four products to be under way
            constexpr int kSums = kN == 1 ? 2 : 1;
            float s[2][kN][4], part[2][kN][4];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int n = 0; n < kN; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[mt][n][e] = part[mt][n][e] = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt) {
                        const uint32_t x = reinterpret_cast<const uint32_t*>(&kx[mt][0][half])[j], y = reinterpret_cast<const uint32_t*>(&kx[mt][1][half])[j];
                        const uint32_t a[4] = {e4m3_low(x), e4m3_low(y), e4m3_high(x), e4m3_high(y)};
#pragma unroll
                        for (int n = 0; n < kN; ++n) mma_h2(half < kSums - 1 ? part[mt][n] : s[mt][n], a, q[n][2 * (4 * half + j)], q[n][2 * (4 * half + j) + 1]);
                    }
            if (kSums > 1) {
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int n = 0; n < kN; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[mt][n][e] += part[mt][n][e];
            }
            if (kN > 1) {
                load_v();
                warp_arrive(bar + Smem::kFree + stage * 8);
            }
            // softmax: weights of V's E4M3 numbers, relative to the largest so far
            float top[kN][2];
            const int32_t left = at.kv - at.tile * 32;     // tokens that there are
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int n = 0; n < kN; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[mt][n][e] = fmaf(s[mt][n][e] * by[mt][e >> 1].x, o.scale_log2, by[mt][e >> 1].y);        // (2^k * scale may leave fp32, and 0 be NaN)
            if (at.tile >= tile_of_masks) {                // some row does not see all of the tile
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int n = 0; n < kN; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (at.tile * 32 + mt * 16 + (e >> 1) * 8 + static_cast<int32_t>(g) >= seen[n][e & 1]) s[mt][n][e] = -INFINITY;
            }
            // The reference m is a row's largest when it was last taken; another one is taken only when a lane has one that is more than 2^8 larger
            // (the weights stand at 2^7 times what they are, at most 2^15), so mostly one vote is all that the lanes need of one another.
            bool grow = false;
#pragma unroll
            for (int n = 0; n < kN; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    top[n][e] = fmaxf(max3(s[0][n][e], s[0][n][2 + e], s[1][n][e]), s[1][n][2 + e]);
                    grow = grow || top[n][e] > m[n][e] + kLazyLog2;            // -inf + 8 is -inf
                }
            if (__any_sync(full, grow)) {
#pragma unroll
                for (int n = 0; n < kN; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float t = top[n][e];
                        t = fmaxf(t, __shfl_xor_sync(full, t, 4));
                        t = fmaxf(t, __shfl_xor_sync(full, t, 8));
                        t = max3(t, __shfl_xor_sync(full, t, 16), m[n][e]);
                        const float by = exp2_fast(m[n][e] - (t == -INFINITY ? 0.0f : t));
                        l[n][e] *= by;
#pragma unroll
                        for (int j = 0; j < 8; ++j) { acc[j][n][e] *= by; acc[j][n][2 + e] *= by; }
                        m[n][e] = t;
                    }
            }
            float plus[kN][2];
#pragma unroll
            for (int n = 0; n < kN; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) plus[n][e] = m[n][e] == -INFINITY ? 0.0f : kManyWeightLog2 - m[n][e];
            uint32_t w[2][kN][2];                          // of sixteen tokens and eight rows each, as the second operand
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int n = 0; n < kN; ++n)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float p[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            p[e] = exp2_fast(s[mt][n][2 * h + e] + plus[n][e]);
                            l[n][e] = fmaf(p[e], by[mt][h].z, l[n][e]);
                        }
                        w[mt][n][h] = turn_8x8(pack_h2(p[0], p[1]));
                    }
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                uint4(&x)[4] = vx[kt];
                if (left < 32) {                           // places behind the last token: whatever is there, nobody sees it
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (static_cast<int32_t>(kt * 16 + 2 * c + (i & 1) + (i >> 1) * 8) >= left) x[i] = make_uint4(0u, 0u, 0u, 0u);
                }
                const uint32_t* const x0 = reinterpret_cast<const uint32_t*>(&x[0]);
                const uint32_t* const x1 = reinterpret_cast<const uint32_t*>(&x[1]);
                const uint32_t* const x2 = reinterpret_cast<const uint32_t*>(&x[2]);
                const uint32_t* const x3 = reinterpret_cast<const uint32_t*>(&x[3]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {              // output dims 16 g + 2 j, 16 g + 2 j + 1
                    const uint32_t sel = j & 1 ? 0x7362u : 0x5140u;
                    const uint32_t near = prmt(x0[j >> 1], x1[j >> 1], sel), far = prmt(x2[j >> 1], x3[j >> 1], sel);
                    const uint32_t a[4] = {e4m3_low(near), e4m3_high(near), e4m3_low(far), e4m3_high(far)};
#pragma unroll
                    for (int n = 0; n < kN; ++n) mma_h2(acc[j][n], a, w[kt][n][0], w[kt][n][1]);
                }
            }
        }
        if (!ok) break;
        // out, or to be joined
        const bool whole = at.begin >= u0 && at.begin + at.units <= u1;
        const int which = from_u == u0 ? 0 : 1;
        float* const to = reinterpret_cast<float*>(which ? smem + (ring - base) : smem + Smem::kFirst + warp * Smem::kPieceBytes);
#pragma unroll
        for (int n = 0; n < kN; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float sum = l[n][e];
                sum += __shfl_xor_sync(full, sum, 4);
                sum += __shfl_xor_sync(full, sum, 8);
                sum += __shfl_xor_sync(full, sum, 16);
                const int row = n * 8 + static_cast<int>(c) * 2 + e;
                if (row >= R) continue;
                if (whole) {
                    const int i = at.group * kP8Rows16 + row, token = i / o.q_per_kv;
                    const int64_t out_row = static_cast<int64_t>(at.row0 + token) * o.q_heads + static_cast<int64_t>(kv.head0 + at.head) * o.q_per_kv + (i - token * o.q_per_kv);
                    const float inv = inverse_of(sum);
                    uint4* const dst = reinterpret_cast<uint4*>(o.out + out_row * kGroup + g * 16);
                    auto two = [&](int j) { return pack_h2(acc[j][n][e] * inv, acc[j][n][2 + e] * inv); };
                    dst[0] = make_uint4(two(0), two(1), two(2), two(3));
                    dst[1] = make_uint4(two(4), two(5), two(6), two(7));
                    if (o.lse && g == 0) o.lse[out_row] = lse_of(m[n][e], sum, kManyWeightLog2);
                } else {
                    float4* const dst = reinterpret_cast<float4*>(to + row * kGroup + g * 16);
#pragma unroll
                    for (int j = 0; j < 4; ++j) dst[j] = make_float4(acc[2 * j][n][e], acc[2 * j][n][2 + e], acc[2 * j + 1][n][e], acc[2 * j + 1][n][2 + e]);
                    if (g == 0) ml[(warp * 2 + which) * kRows + row] = make_float2(m[n][e], sum);
                }
            }
        if (!whole && lane == 0) pieces[warp * 2 + which] = P8Piece{at.begin, at.units, at.head, at.row0, at.rows, at.group, 1};
        seek(at, u1);
    }
    meet();

    auto write_row = [&](int32_t group, int32_t row0, int32_t head, int row, float m, float l, const float4& v) {
        const int i = group * kP8Rows16 + row, token = i / o.q_per_kv;
        const int64_t out_row = static_cast<int64_t>(row0 + token) * o.q_heads + static_cast<int64_t>(kv.head0 + head) * o.q_per_kv + (i - token * o.q_per_kv);
        const float inv = inverse_of(l);
        reinterpret_cast<uint2*>(o.out + out_row * kGroup)[lane] = make_uint2(pack_h2(v.x * inv, v.y * inv), pack_h2(v.z * inv, v.w * inv));
        if (o.lse && lane == 0) o.lse[out_row] = lse_of(m, l, kManyWeightLog2);
    };
    // pieces of the CTA's warps, one behind the other in the line: lane i looks at the i-th of them
    const uint32_t nth = min(lane, 2u * kP8Warps - 1u);
    const int64_t of_lane = pieces[nth].begin;
    const unsigned valid = __ballot_sync(full, lane < 2 * kP8Warps && pieces[nth].valid);
    const unsigned ahead = valid & ((1u << lane) - 1u);
    const int64_t of_ahead = __shfl_sync(full, of_lane, ahead ? 31 - __clz(ahead) : 0);
    unsigned firsts = __ballot_sync(full, (valid >> lane & 1u) && (!ahead || of_ahead != of_lane));
    for (uint32_t first_row = warp; firsts; first_row ^= kP8Warps / 2) {               // pieces of few rows one after the other go to other warps
        const int i = __ffs(firsts) - 1;
        firsts &= firsts - 1u;
        const unsigned members = valid & ~((1u << i) - 1u) & (firsts ? (1u << (__ffs(firsts) - 1)) - 1u : full);
        const P8Piece p = pieces[i];
        const int R = min(p.rows * o.q_per_kv - p.group * kP8Rows16, kN * 8);
        // a warp's rows, of which there are one or two, side by side
        float m[kN], l[kN];
        float4 v[kN];
#pragma unroll
        for (int n = 0; n < kN; ++n) { m[n] = -INFINITY; l[n] = 0.0f; v[n] = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
        for (unsigned left = static_cast<int>(first_row) < R ? members : 0u; left; left &= left - 1u) {
            const int j = __ffs(left) - 1;
            const uint8_t* const from = j & 1 ? smem + Smem::kRing + (j >> 1) * kP8Stages * kP8StageBytes : smem + Smem::kFirst + (j >> 1) * Smem::kPieceBytes;
#pragma unroll
            for (int n = 0; n < kN; ++n) {
                const int row = min(static_cast<int>(first_row) + n * kP8Warps, R - 1);
                join_sums(m[n], l[n], v[n], ml[j * kRows + row], reinterpret_cast<const float4*>(from)[row * 32 + lane]);
            }
        }
#pragma unroll
        for (int n = 0; n < kN; ++n) {
            const int row = static_cast<int>(first_row) + n * kP8Warps;
            if (row >= R) break;
            if (p.begin >= c0 && p.begin + p.units <= c1) {
                write_row(p.group, p.row0, p.head, row, m[n], l[n], v[n]);
            } else {
                const int64_t to = (static_cast<int64_t>(blockIdx.x) * 2 + (p.begin < c0 ? 0 : 1)) * kP8Rows16 + row;
                reinterpret_cast<float4*>(f.part + to * kGroup)[lane] = v[n];
                if (lane == 0) f.part_ml[to] = make_float2(m[n], l[n]);
            }
        }
    }
    if (o.early) dependency_wait();
    if (f.by_request) return;
    if (!spans[0].valid && !spans[1].valid) return;
    meet();
    if (tid < 2) {
        const P8Span sp = spans[tid];
        __threadfence();                                   // what all threads have written before the barrier
        joins[tid] = sp.valid && take_ticket(f.tickets + static_cast<int64_t>(sp.lo) * kTicketStride) == static_cast<unsigned>(sp.hi - sp.lo);
        __threadfence();
    }
    meet();
    for (int i = 0; i < 2; ++i) {
        if (!joins[i]) continue;
        const P8Span sp = spans[i];
        const int R = min(sp.rows * o.q_per_kv - sp.group * kP8Rows16, kN * 8);
        const int first_row = static_cast<int>(warp ^ (i ? kP8Warps / 2 : 0));
        float m[kN], l[kN];
        float4 v[kN];
#pragma unroll
        for (int n = 0; n < kN; ++n) { m[n] = -INFINITY; l[n] = 0.0f; v[n] = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
        for (int b0 = sp.lo; b0 <= sp.hi && first_row < R; b0 += 8) {                  // eight pieces on their way together
            float2 x[8][kN];
            float4 y[8][kN];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int b = min(b0 + k, sp.hi);
#pragma unroll
                for (int n = 0; n < kN; ++n) {
                    const int64_t from = (static_cast<int64_t>(b) * 2 + (sp.begin < cta_split.begin(b) ? 0 : 1)) * kP8Rows16 + min(first_row + n * kP8Warps, R - 1);
                    x[k][n] = __ldcg(f.part_ml + from);
                    y[k][n] = __ldcg(reinterpret_cast<const float4*>(f.part + from * kGroup) + lane);
                }
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (b0 + k <= sp.hi)
#pragma unroll
                    for (int n = 0; n < kN; ++n) join_sums(m[n], l[n], v[n], x[k][n], y[k][n]);
        }
#pragma unroll
        for (int n = 0; n < kN; ++n)
            if (first_row + n * kP8Warps < R) write_row(sp.group, sp.row0, sp.head, first_row + n * kP8Warps, m[n], l[n], v[n]);
        if (tid == 0) *(f.tickets + static_cast<int64_t>(sp.lo) * kTicketStride) = 0;
    }
}

}  // namespace
