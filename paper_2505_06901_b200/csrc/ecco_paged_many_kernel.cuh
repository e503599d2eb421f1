// ecco_paged_many_kernel.cuh -- K6m: attention of requests of many rows over a paged KV cache, on tcgen05
// Part of the one translation unit ecco_kernels.cu; included from there only.
#pragma once

namespace {

// ---------------------------------------------------------------------------------------------
// K6m: pieces of prompts: a request's rows (new tokens x query heads per KV head, query heads innermost) in blocks of 256.
//   S = Q K^T    128 x 128 per tile of rows and tile of tokens; Q and K from shared memory, S to tensor memory
//   P = 2^(scale S - m)   in registers, a thread to a row; fp16, back to tensor memory over S
//   O += P V     P from tensor memory, V from shared memory, O in tensor memory
// Two tiles of rows share every K and V tile, and while one's products run, the other's softmax does.
// Warps 0-3 and 4-7: softmax of the first and of the second tile of rows; warp 8: loads; warp 9: one thread issues the products.
// m is the row's maximum when it was last taken; a larger one is taken only when it is more than 2^8 larger (the weights are fp16
// times 2^7, at most 2^15), so O is rescaled now and then instead of with every tile.
//
// All blocks' tiles of all heads form one line, which is cut into equal runs, one per CTA (see paged_schedule): a block that is cut leaves
// its sums in the workspace and ecco_paged_join_kernel joins them.
// ---------------------------------------------------------------------------------------------
constexpr int kManyThreads = 384;                          // warps 10 and 11 only give their registers away
constexpr uint32_t kOperandBytes = 8 * 4096;               // eight pieces of [128][16] fp16, 32-byte swizzle
constexpr int kManyStages = 5;                             // tiles of K and V in flight
constexpr uint32_t kManySmemBytes = 1024 + (2 + kManyStages) * kOperandBytes;
static_assert(kManySmemBytes <= kSmemCtaBytes, "fits an SM");
constexpr float kManyWeightLog2 = 7.0f, kLazyLog2 = 8.0f;

__device__ __forceinline__ void tmem_ld32(uint32_t* r, uint32_t at)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                   "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]),
                   "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(at));
}
__device__ __forceinline__ void tmem_st32(uint32_t at, const uint32_t* r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
                 ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
                 "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
                 "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
                 : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
// arrives when all products issued so far by this thread are done
__device__ __forceinline__ void mma_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Shared-memory operand with 32-byte swizzle: rows of 32 bytes, blocks of eight rows `stride` bytes apart; `lead`: what is 16 elements on
// in the direction of the rows' bytes, where the operand is wider than that (MN-major only).
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t lead, uint32_t stride)
{
    return static_cast<uint64_t>((at & 0x3ffffu) >> 4) | (static_cast<uint64_t>(lead >> 4) << 16) | (static_cast<uint64_t>(stride >> 4) << 32) | (1ull << 46) | (6ull << 61);
}
// 128 x 128 x 16, fp16 x fp16 -> fp32; b_mn: B's contiguous direction is N
__host__ __device__ constexpr uint32_t mma_shape(bool b_mn) { return (1u << 4) | (b_mn ? 1u << 16 : 0u) | ((128u >> 3) << 17) | ((128u >> 4) << 24); }
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, bool add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(shape),
                 "r"(static_cast<uint32_t>(add))
                 : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t shape, bool add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(shape),
                 "r"(static_cast<uint32_t>(add))
                 : "memory");
}

// a piece of a block: tiles [from, to) of the `tiles` tiles of block `block` of request r, for head `head`
struct ManyPiece { int64_t next; int32_t head, r, block, tiles, from, to; };
__device__ __forceinline__ ManyPiece many_piece(const PagedSchedule& sc, int32_t n_blocks, int64_t total, int64_t u, int64_t u1)
{
    ManyPiece p;
    p.head = static_cast<int32_t>(divide(static_cast<uint64_t>(u), static_cast<uint64_t>(total)));
    const int32_t at = static_cast<int32_t>(u - p.head * total);
    const int j = warp_find(sc.block_tiles, n_blocks, at);
    const int32_t first = __ldcg(sc.block_tiles + j), end = __ldcg(sc.block_tiles + j + 1);
    const int2 rb = __ldcg(sc.blocks + j);
    p.r = rb.x;
    p.block = rb.y;
    p.tiles = end - first;
    p.from = at - first;
    p.to = static_cast<int32_t>(min(static_cast<int64_t>(p.tiles), p.from + (u1 - u)));
    p.next = u + (p.to - p.from);
    return p;
}

__global__ void __launch_bounds__(kManyThreads, 1)
ecco_paged_many_kernel(const __grid_constant__ PagedKv kv, const __grid_constant__ PagedOut o, const __grid_constant__ PagedSchedule sc)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, base = smem_u32(smem);
    // barriers: tiles have come / are free again, Q there, S there, P there, O there
    const uint32_t full_at = base, free_at = base + 8 * kManyStages, q_bar = base + 128, s_bar = base + 144, p_bar = base + 160, o_bar = base + 176, end_bar = base + 192;
    const uint32_t q_smem = base + 1024, ring = q_smem + 2 * kOperandBytes;
    uint32_t* const tmem_word = reinterpret_cast<uint32_t*>(smem + 256);
    volatile int* const failed = reinterpret_cast<volatile int*>(smem + 264);
    if (threadIdx.x == 0) {
        for (int i = 0; i < kManyStages; ++i) { mbar_init(full_at + 8 * i, 1); mbar_init(free_at + 8 * i, 1); }
        for (int x = 0; x < 2; ++x) { mbar_init(q_bar + 8 * x, 128); mbar_init(s_bar + 8 * x, 1); mbar_init(p_bar + 8 * x, 128); mbar_init(o_bar + 8 * x, 1); }
        mbar_init(end_bar, 1);
        *failed = 0;
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(tmem_word)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        tmem_fence_before();
    }
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = *tmem_word;                      // columns 0, 128: S and P; 256, 384: O
    dependency_wait();
    release_dependents();
    const int32_t n_blocks = __ldcg(sc.n_blocks), total = n_blocks > 0 ? __ldcg(sc.block_tiles + n_blocks) : 0;
    const UnitSplit split(static_cast<int64_t>(total) * kv.heads, static_cast<int>(gridDim.x));
    const int64_t u0 = split.begin(static_cast<int>(blockIdx.x)), u1 = split.begin(static_cast<int>(blockIdx.x) + 1);
    const int32_t T = paged_tiles(kv);
    const bool causal = o.causal;
    // a wait that has run out makes all others run out at once
    auto wait = [&](uint32_t bar, uint32_t parity) {
        bool done = false;
        for (int i = 0; i < 2 * kWaitLimit && !done; ++i) {
            done = mbar_try_wait(bar, parity);
            if (!done && (i & 63) == 63 && *failed) break;
        }
        if (!done) { *failed = 1; atomicExch(&g_device_status, ECCO_ERR_DEVICE_TIMEOUT); }
        return done;
    };

    // 384 threads x 168 registers = 128 x 40 + 256 x 232
    if (warp >= 8) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    else asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
    if (warp < 8) {
        // softmax: thread t of tile x holds row 128 x + t
        const uint32_t x = warp >> 2, t = threadIdx.x & 127u, s_at = tmem + ((warp & 3u) << 21) + x * 128, o_at = s_at + 256;
        uint32_t n_s = 0, n_o = 0;                         // S and O waited for
        bool ok = true;
        for (int64_t u = u0; u < u1 && ok;) {
            const ManyPiece pc = many_piece(sc, n_blocks, total, u, u1);
            const PagedReq q = paged_req(kv, pc.r, T);
            const int slot = 2 * static_cast<int>(blockIdx.x) + (u == u0 ? 0 : 1);
            u = pc.next;
            const int64_t rows = static_cast<int64_t>(q.rows) * o.q_per_kv, row = static_cast<int64_t>(pc.block) * kManyRows + x * 128 + t;
            if (x == 1 && rows <= static_cast<int64_t>(pc.block) * kManyRows + 128) continue;             // one tile of rows only
            const bool exists = row < rows;
            const int32_t token = static_cast<int32_t>((exists ? row : 0) / o.q_per_kv), g = static_cast<int32_t>(row - static_cast<int64_t>(token) * o.q_per_kv);
            const int64_t out_row = static_cast<int64_t>(q.row0 + token) * o.q_heads + (kv.head0 + pc.head) * o.q_per_kv + g;
            const int32_t seen = exists ? tokens_seen(q, token, causal) : 0;
            {
                // a negative scale is taken as its size, with q negated
                const uint4* const src = reinterpret_cast<const uint4*>(o.q + (q.row0 + token) * o.q_stride + (static_cast<int64_t>(kv.head0 + pc.head) * o.q_per_kv + g) * kGroup);
                const uint32_t flip = o.scale_log2 < 0.0f ? 0x80008000u : 0u, dst = q_smem + x * kOperandBytes + t * 32;
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    uint4 v = make_uint4(0u, 0u, 0u, 0u);
                    if (exists) v = __ldcg(src + c);
                    sts_v4(dst + (c >> 1) * 4096 + (((c & 1) ^ ((t >> 2) & 1u)) << 4), v.x ^ flip, v.y ^ flip, v.z ^ flip, v.w ^ flip);
                }
                fence_async_smem();
                mbar_arrive(q_bar + 8 * x);
            }
            const float scale = fabsf(o.scale_log2);
            float m = -INFINITY, l = 0.0f;                 // m in units of log2, the weights stand at 2^(s - m + kManyWeightLog2)
            for (int32_t j = pc.from; j < pc.to; ++j) {
                ok = wait(s_bar + 8 * x, n_s++ & 1u);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                tmem_fence_after();
                float s[128];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(reinterpret_cast<uint32_t*>(s) + 32 * c, s_at + 32 * c);
                tmem_wait_ld();
                const int32_t left = seen - j * kManyTokens;           // columns that the row sees
                if (__any_sync(0xffffffffu, left < kManyTokens)) {
#pragma unroll
                    for (int c = 0; c < 128; ++c) s[c] = c < left ? s[c] : -INFINITY;
                }
                float top = s[0];
#pragma unroll
                for (int c = 1; c < 128; ++c) top = fmaxf(top, s[c]);
                top *= scale;
                if (left <= 0) top = -INFINITY;            // also where the scale is zero
                const bool grow = top > m + kLazyLog2;     // -inf + 8 is -inf
                if (__any_sync(0xffffffffu, grow)) {
                    const float m_new = grow ? top : m, f = grow ? exp2_fast(m - top) : 1.0f;
                    m = m_new;
                    l *= f;
                    if (j > pc.from) {                     // the products of the tile before are done: S of this one came behind them
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            uint32_t v[32];
                            tmem_ld32(v, o_at + 32 * c);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * f);
                            tmem_st32(o_at + 32 * c, v);
                        }
                    }
                }
                const float sub = kManyWeightLog2 - (m == -INFINITY ? 0.0f : m);
                float sum0 = 0.0f, sum1 = 0.0f;
                uint32_t p[64];
#pragma unroll
                for (int c = 0; c < 64; ++c) {
                    const float a = exp2_fast(fmaf(s[2 * c], scale, sub)), b = exp2_fast(fmaf(s[2 * c + 1], scale, sub));
                    sum0 += a;
                    sum1 += b;
                    p[c] = pack_h2(a, b);
                }
                l += sum0 + sum1;
                tmem_st32(s_at, p);
                tmem_st32(s_at + 32, p + 32);
                tmem_wait_st();
                tmem_fence_before();
                mbar_arrive(p_bar + 8 * x);
            }
            if (!ok) break;
            ok = wait(o_bar + 8 * x, n_o++ & 1u);
            if (!__all_sync(0xffffffffu, ok)) break;
            tmem_fence_after();
            const bool whole = pc.from == 0 && pc.to == pc.tiles;
            const float inv = l > 0.0f ? 1.0f / l : 0.0f;
            float* const part = o.part + (static_cast<int64_t>(slot) * kManyRows + x * 128 + t) * kGroup;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t v[32];
                tmem_ld32(v, o_at + 32 * c);
                tmem_wait_ld();
                if (exists && whole) {
                    uint4* const dst = reinterpret_cast<uint4*>(o.out + out_row * kGroup) + 4 * c;
                    // a row that has seen nothing: O may not have been written at all
                    auto two = [&](int i) { return l > 0.0f ? pack_h2(__uint_as_float(v[i]) * inv, __uint_as_float(v[i + 1]) * inv) : 0u; };
#pragma unroll
                    for (int i = 0; i < 4; ++i) dst[i] = make_uint4(two(8 * i), two(8 * i + 2), two(8 * i + 4), two(8 * i + 6));
                } else if (exists) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) reinterpret_cast<uint4*>(part)[8 * c + i] = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                }
                __syncwarp();
            }
            if (exists) {
                if (whole) { if (o.lse) o.lse[out_row] = lse_of(m, l, kManyWeightLog2); }
                else o.part_ml[static_cast<int64_t>(slot) * kManyRows + x * 128 + t] = make_float2(m, l);
            }
            tmem_fence_before();                           // O has been read before the next block's P arrives
        }
    } else if (warp == 8) {
        // loads: K and V tiles in the order in which they are used
        uint32_t n = 0;
        bool ok = true;
        for (int64_t u = u0; u < u1 && ok;) {
            const ManyPiece pc = many_piece(sc, n_blocks, total, u, u1);
            const PagedReq q = paged_req(kv, pc.r, T);
            u = pc.next;
            for (int32_t j = pc.from; j < pc.to && ok; ++j) {
                const int32_t tiles = min(max(q.tiles - 4 * j, 0), 4);         // of 32 tokens
                for (int which = 0; which < 2; ++which) {
                    const uint32_t st = n % kManyStages, bar = full_at + 8 * st, dst = ring + st * kOperandBytes;
                    if (n >= kManyStages) ok = __all_sync(0xffffffffu, wait(free_at + 8 * st, (n / kManyStages - 1) & 1u));
                    if (!ok) break;
                    ++n;
                    if (lane == 0) mbar_expect_tx(bar, tiles * kKvTileBytes);
                    __syncwarp();
                    // piece lane % 8 of tile lane / 8
                    if (static_cast<int32_t>(lane >> 3) < tiles)
                        bulk_g2s(dst + (lane & 7u) * 4096 + (lane >> 3) * kPieceBytes,
                                 staged_tile(kv, which, pc.head, q.first + 4 * j + static_cast<int32_t>(lane >> 3)) + (lane & 7u) * kPieceBytes, kPieceBytes, bar);
                }
            }
        }
        if (!ok)                                           // what is on its way lands before the CTA leaves
            for (uint32_t i = n < kManyStages ? 0 : n - kManyStages; i < n; ++i)
                for (int k = 0; k < kWaitLimit && !mbar_try_wait(full_at + 8 * (i % kManyStages), (i / kManyStages) & 1u); ++k) {}
    } else if (warp == 9) {
        // products: one thread issues them
        uint32_t n = 0, n_q[2] = {0, 0}, n_p[2] = {0, 0};
        bool ok = true;
        for (int64_t u = u0; u < u1 && ok;) {
            const ManyPiece pc = many_piece(sc, n_blocks, total, u, u1);
            const PagedReq q = paged_req(kv, pc.r, T);
            u = pc.next;
            const int n_x = static_cast<int64_t>(q.rows) * o.q_per_kv > static_cast<int64_t>(pc.block) * kManyRows + 128 ? 2 : 1;
            if (lane == 0) {
                auto scores = [&](int x, uint32_t st) {
#pragma unroll
                    for (int d = 0; d < 8; ++d)
                        mma_ss(tmem + x * 128, operand(q_smem + x * kOperandBytes + d * 4096, 16, 256), operand(ring + st * kOperandBytes + d * 4096, 16, 256), mma_shape(false), d > 0);
                    mma_commit(s_bar + 8 * x);
                };
                auto come = [&](uint32_t i) {
                    ok = ok && wait(full_at + 8 * (i % kManyStages), (i / kManyStages) & 1u);
                    return i % kManyStages;
                };
                uint32_t k_st = come(n);
                for (int x = 0; x < n_x && ok; ++x) {
                    ok = wait(q_bar + 8 * x, n_q[x]++ & 1u);
                    tmem_fence_after();
                    if (ok) scores(x, k_st);
                }
                if (ok) mma_commit(free_at + 8 * k_st);
                for (int32_t j = pc.from; j < pc.to && ok; ++j) {
                    const bool more = j + 1 < pc.to;
                    const uint32_t v_st = come(n + 1);
                    n += 2;
                    // sixteen tokens at a time, as far as there are tiles
                    const int steps = min(max(q.tiles - 4 * j, 0), 4) * 2;
                    for (int x = 0; x < n_x && ok; ++x) {
                        ok = wait(p_bar + 8 * x, n_p[x]++ & 1u);
                        if (!ok) break;
                        tmem_fence_after();
                        for (int ks = 0; ks < steps; ++ks)
                            mma_ts(tmem + 256 + x * 128, tmem + x * 128 + ks * 8, operand(ring + v_st * kOperandBytes + ks * 512, 4096, 256), mma_shape(true), j > pc.from || ks > 0);
                        if (x == n_x - 1) mma_commit(free_at + 8 * v_st);
                        if (more) {
                            if (x == 0) k_st = come(n);
                            if (ok) scores(x, k_st);
                            if (x == n_x - 1) mma_commit(free_at + 8 * k_st);
                        } else {
                            mma_commit(o_bar + 8 * x);
                        }
                    }
                }
                if (!ok) {                                 // what has been issued ends before tensor memory is given back
                    mma_commit(end_bar);
                    for (int k = 0; k < kWaitLimit && !mbar_try_wait(end_bar, 0); ++k) {}
                }
            }
            ok = __shfl_sync(0xffffffffu, ok, 0);
            __syncwarp();
        }
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

// Joins the pieces of blocks that were cut: CTA (c, part) looks at the cut in front of run c, and if it is its block's first one
// joins 32 of the block's rows.  A warp to a row.
constexpr int kJoinParts = kManyRows / 32;
__global__ void __launch_bounds__(256)
ecco_paged_join_kernel(const __grid_constant__ PagedKv kv, const __grid_constant__ PagedOut o, const __grid_constant__ PagedSchedule sc, int many_ctas)
{
    release_dependents();
    const int c = static_cast<int>(blockIdx.x) / kJoinParts + 1, part = static_cast<int>(blockIdx.x) % kJoinParts;
    const int lane = static_cast<int>(threadIdx.x & 31u), warp = static_cast<int>(threadIdx.x >> 5);
    dependency_wait();
    const int32_t n_blocks = __ldcg(sc.n_blocks), total = n_blocks > 0 ? __ldcg(sc.block_tiles + n_blocks) : 0;
    const int64_t U = static_cast<int64_t>(total) * kv.heads;
    const UnitSplit split(U, many_ctas);
    const int64_t cut = split.begin(c);
    if (cut >= U) return;
    const ManyPiece pc = many_piece(sc, n_blocks, total, cut, U);
    const int64_t first = cut - pc.from, end = first + pc.tiles;
    if (pc.from == 0 || split.begin(c - 1) > first) return;        // not inside of a block, or not its first cut
    const int w_lo = c - 1, w_hi = split.owner(end - 1);
    const bool second = split.begin(w_lo) != first;        // the piece in run w_lo is in its second slot
    const PagedReq q = paged_req(kv, pc.r, paged_tiles(kv));
    for (int i = warp; i < 32; i += 8) {
        const int in_block = part * 32 + i;
        const int64_t row = static_cast<int64_t>(pc.block) * kManyRows + in_block;
        if (row >= static_cast<int64_t>(q.rows) * o.q_per_kv) return;
        float m = -INFINITY, l = 0.0f;
        float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int w = w_lo; w <= w_hi; ++w) {
            const int64_t at = (2 * static_cast<int64_t>(w) + (w == w_lo && second ? 1 : 0)) * kManyRows + in_block;
            const float2 x = __ldcg(o.part_ml + at);
            const float4 v = __ldcg(reinterpret_cast<const float4*>(o.part + at * kGroup) + lane);
            join_sums(m, l, acc, x, v);
        }
        const int32_t token = static_cast<int32_t>(row / o.q_per_kv), g = static_cast<int32_t>(row - static_cast<int64_t>(token) * o.q_per_kv);
        const int64_t out_row = static_cast<int64_t>(q.row0 + token) * o.q_heads + (kv.head0 + pc.head) * o.q_per_kv + g;
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        reinterpret_cast<uint2*>(o.out + out_row * kGroup)[lane] = make_uint2(pack_h2(acc.x * inv, acc.y * inv), pack_h2(acc.z * inv, acc.w * inv));
        if (o.lse && lane == 0) o.lse[out_row] = lse_of(m, l, kManyWeightLog2);
    }
}

}  // namespace
