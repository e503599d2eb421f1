// ecco_paged_many_kernel.cuh -- K6m: attention of requests of many rows over a paged KV cache, on tcgen05
// Part of the one translation unit ecco_kernels.cu; included from there only.
#pragma once

namespace {

// ---------------------------------------------------------------------------------------------
// K6m: pieces of prompts: a request's rows (new tokens x query heads per KV head, query heads innermost) in blocks of 256.
// (as many whole tokens as two tiles of 128 rows hold)
//   S = Q K^T    128 x 128 per tile of rows and tile of tokens; Q and K from shared memory, S to tensor memory
//   P = 2^(scale S - m)   in registers, a thread to a row; fp16, back to tensor memory over S
//   O += P V     P from tensor memory, V from shared memory, O in tensor memory
// Two tiles of rows share every K and V tile, and while one's products run, the other's softmax does.
// Warps 0-3 and 4-7: softmax of the first and of the second tile of rows; warp 8: K and V; warp 9 issues the
// products; warp 10: Q, and what there is to do (ManyTask); warp 11 only gives its registers away.
// What carries it: operands that lie in uniform registers, waits that one vote decides (see below), weights sent in two halves, the
// next block's Q and first scores under way while this one's sums are written out.  A tile of tokens takes two tiles of rows some 3100 clocks,
// 2048 of them products: a thread's softmax (1.7 thousand clocks, 128 exponentials in it) and the products behind its last weights follow
// one another.  2 x 2048 tokens x 32 heads over 8000 tokens, 468 GFLOP: some 385 us = 1.2 PFLOP/s in a burst of calls (a
// call over E4M3 numbers, 406 us, less the 22 that make the tiles); a second of them takes an eighth longer, the power limit holding the SMs at 1.65 of 1.965 GHz.
// (Measured equal or slower: the maximum searched for beside the first weights, an eighth or a quarter of the exponentials as polynomials, a warp
// of products for each tile of rows, the tokens of a block of one tile of rows shared out between both tiles' warps.)
// m is the row's maximum when it was last taken; a larger one is taken only when it is more than 2^8 larger (the weights are fp16
// times 2^7, at most 2^15), so O is rescaled now and then instead of with every tile.
//
// All blocks' tiles of all heads form one line, which is cut into equal runs, one per CTA (see paged_schedule).  A block that is cut leaves
// its sums in the workspace, and whoever comes last joins them, in the order of the runs.
// ---------------------------------------------------------------------------------------------
constexpr uint32_t kOperandBytes = 8 * 4096;               // eight pieces of [128][16] fp16, 32-byte swizzle
// k8: K and V come as E4M3 numbers from the pages of a cache in 8 bits (ecco_paged8_kernels.cuh), and four more warps make the tiles of them, a thread to a token: 16
// bytes of shared memory become 32, exactly, with the token's power of two multiplied in.  With 64 KB more through shared memory, whose pipe is busy for two
// thirds of the time as it is, a tile of tokens takes a sixth longer; tiles made beforehand (K8s) cost as much as nine blocks lose by that.
constexpr uint32_t kCodeBytes = 128 * kGroup;              // an operand as E4M3 numbers
constexpr int kCodeStages = 2;
template <bool k8> struct ManyShape {
    static constexpr int kThreads = k8 ? 512 : 384;
    static constexpr int kStages = k8 ? 4 : 5;             // tiles of K and V in flight
    static constexpr uint32_t kCodes = 1024 + (2 + kStages) * kOperandBytes, kWords = kCodes + kCodeStages * kCodeBytes;
    static constexpr uint32_t kBytes = k8 ? kWords + kCodeStages * 128 * 8 : kCodes;
    static_assert(kBytes <= kSmemCtaBytes, "fits an SM");
};
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
// what was loaded is used behind this point only: the compiler does not see that the wait in front concerns these registers
__device__ __forceinline__ void tie32(uint32_t* r)
{
    asm volatile("" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]),
                      "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]),
                      "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]));
    asm volatile("" : "+r"(r[29]), "+r"(r[30]), "+r"(r[31]));
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// one arrival for the whole warp (32 at one address go one after the other)
__device__ __forceinline__ void warp_arrive(uint32_t bar)
{
    __syncwarp();
    if ((threadIdx.x & 31u) == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// by a converged warp: arrives when all products that it has issued so far are done
__device__ __forceinline__ void mma_commit(uint32_t bar)
{
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\t@p tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar) : "memory");
}
// two fp32 operations in one instruction
__device__ __forceinline__ uint64_t pack_f2(float a, float b)
{
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    return v;
}
__device__ __forceinline__ void unpack_f2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma_f2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t v;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
    return v;
}
__device__ __forceinline__ uint64_t mul_f2(uint64_t a, uint64_t b)
{
    uint64_t v;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
    return v;
}
__device__ __forceinline__ uint64_t add_f2(uint64_t a, uint64_t b)
{
    uint64_t v;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
    return v;
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float v;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(v) : "f"(a), "f"(b), "f"(c));
    return v;
}
// Shared-memory operand with 32-byte swizzle: rows of 32 bytes, blocks of eight rows `stride` bytes apart; `lead`: what is 16 elements on
// in the direction of the rows' bytes, where the operand is wider than that (MN-major only).
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t lead, uint32_t stride)
{
    return static_cast<uint64_t>((at & 0x3ffffu) >> 4) | (static_cast<uint64_t>(lead >> 4) << 16) | (static_cast<uint64_t>(stride >> 4) << 32) | (1ull << 46) | (6ull << 61);
}
// 128 x 128 x 16, fp16 x fp16 -> fp32; b_mn: B's contiguous direction is N
__host__ __device__ constexpr uint32_t mma_shape(bool b_mn) { return (1u << 4) | (b_mn ? 1u << 16 : 0u) | ((128u >> 3) << 17) | ((128u >> 4) << 24); }
// One lane of a converged warp issues the products; what they get as operands has to be the same in all lanes, and known to the compiler
// to be (see same_in_warp): it lies in uniform registers then, and an instruction takes as long to issue as the tensor core takes to do
// it.  With one lane in a branch of its own it was some 130 clocks against 64.
__device__ __forceinline__ int same_in_warp(int v) { return __reduce_max_sync(0xffffffffu, v); }
// S = Q K^T of a tile: eight steps of 16 dims, 4096 bytes apart in both operands
__device__ __forceinline__ void mma_scores(uint32_t d, uint64_t a, uint64_t b)
{
    asm volatile(
        "{\n\t.reg .pred p, f, t;\n\t.reg .b64 a, b;\n\telect.sync _|p, 0xffffffff;\n\tsetp.ne.u32 f, 0, 0;\n\tsetp.eq.u32 t, 0, 0;\n\tmov.b64 a, %1;\n\tmov.b64 b, %2;\n\t"
        "@p tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, f;\n\t"
        "add.u64 a, a, 256;\n\tadd.u64 b, b, 256;\n\t@p tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n\t"
        "add.u64 a, a, 256;\n\tadd.u64 b, b, 256;\n\t@p tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n\t"
        "add.u64 a, a, 256;\n\tadd.u64 b, b, 256;\n\t@p tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n\t"
        "add.u64 a, a, 256;\n\tadd.u64 b, b, 256;\n\t@p tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n\t"
        "add.u64 a, a, 256;\n\tadd.u64 b, b, 256;\n\t@p tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n\t"
        "add.u64 a, a, 256;\n\tadd.u64 b, b, 256;\n\t@p tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n\t"
        "add.u64 a, a, 256;\n\tadd.u64 b, b, 256;\n\t@p tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(mma_shape(false))
        : "memory");
}
// O (+)= P V over 64 tokens: four steps, eight columns of P and 512 bytes of V apart
__device__ __forceinline__ void mma_values4(uint32_t d, uint32_t a, uint64_t b, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p, q, t;\n\t.reg .b32 a;\n\t.reg .b64 b;\n\telect.sync _|p, 0xffffffff;\n\tsetp.ne.u32 q, %4, 0;\n\tsetp.eq.u32 t, 0, 0;\n\tmov.b32 a, %1;\n\tmov.b64 b, %2;\n\t"
        "@p tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, q;\n\t"
        "add.u32 a, a, 8;\n\tadd.u64 b, b, 32;\n\t@p tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n\t"
        "add.u32 a, a, 8;\n\tadd.u64 b, b, 32;\n\t@p tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n\t"
        "add.u32 a, a, 8;\n\tadd.u64 b, b, 32;\n\t@p tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(mma_shape(true)), "r"(static_cast<uint32_t>(add))
        : "memory");
}
// the same over 16 tokens
__device__ __forceinline__ void mma_values(uint32_t d, uint32_t a, uint64_t b, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\telect.sync _|p, 0xffffffff;\n\tsetp.ne.u32 q, %4, 0;\n\t@p tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, q;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(mma_shape(true)), "r"(static_cast<uint32_t>(add))
        : "memory");
}

// a piece of a block: tiles [from, to) of the `tiles` tiles of block `block` of request r, for head `head`
struct ManyPiece { int64_t next; int32_t head, r, block, tiles, from, to; };
__device__ __forceinline__ ManyPiece many_piece(const PagedSchedule& sc, int32_t heads, int32_t n_blocks, int64_t total, int64_t u, int64_t u1)
{
    ManyPiece p;
    const int32_t nth = static_cast<int32_t>(divide(static_cast<uint64_t>(u), static_cast<uint64_t>(total)));
    const int32_t at = static_cast<int32_t>(u - nth * total);
    p.head = heads - 1 - nth;                              // the last head's tiles are the latest in the L2 cache
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

// what the other warps need to know of a piece, for a tile of its rows (read from shared memory)
struct ManyTask {
    int32_t used;              // the tile has rows
    int32_t from, to, tiles;   // of 128 tokens; of 32 tokens: the request's
    int32_t head, r_row0, r_rows, r_kv;   // KV head, the request's rows of q and tokens
    int32_t token;             // the tile's first new token of the request
    int32_t whole, slot;       // the piece is its block; else: place of its sums,
    int32_t run_lo, run_hi, second;    // the runs that have pieces of the block; the first of them has it in its second slot
};

// k_map: the tiles; k8: the pool of K
template <bool k8>
__global__ void __launch_bounds__(ManyShape<k8>::kThreads, 1)
ecco_paged_many_kernel(const __grid_constant__ PagedKv kv, const __grid_constant__ PagedOut o, const __grid_constant__ PagedSchedule sc,
                       const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const __grid_constant__ CUtensorMap q_map)
{
    constexpr int kManyStages = ManyShape<k8>::kStages;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, base = smem_u32(smem);
    // barriers: tiles have come / are free again, Q there, S there, P there, O there
    const uint32_t code_at = base + 80, code_free = code_at + 8 * kCodeStages;         // k8: numbers have come / have been read
    const uint32_t full_at = base, free_at = base + 8 * kManyStages, q_bar = base + 128, s_bar = base + 144, p_bar = base + 160 /* halves, tiles of rows */, o_bar = base + 192, q_free = base + 208, end_bar = base + 224, in_bar = base + 272, told_bar = base + 288;
    const uint32_t q_smem = base + 1024, ring = q_smem + 2 * kOperandBytes;
    uint32_t* const tmem_word = reinterpret_cast<uint32_t*>(smem + 256);
    volatile int* const failed = reinterpret_cast<volatile int*>(smem + 264);
    ManyTask* const tasks = reinterpret_cast<ManyTask*>(smem + 320);       // [two pieces][tile of rows]
    static_assert(320 + 4 * sizeof(ManyTask) <= 1008, "tasks fit");
    volatile int* const last_in = reinterpret_cast<volatile int*>(smem + 1008);          // [tile of rows]
    if (threadIdx.x == 0) {
        for (int i = 0; i < kManyStages; ++i) { mbar_init(full_at + 8 * i, k8 ? 4 : 1); mbar_init(free_at + 8 * i, 1); }
        if (k8)
            for (int i = 0; i < kCodeStages; ++i) { mbar_init(code_at + 8 * i, 33); mbar_init(code_free + 8 * i, 4); }
        for (int x = 0; x < 2; ++x) { mbar_init(q_bar + 8 * x, 1); mbar_init(q_free + 8 * x, 5); mbar_init(s_bar + 8 * x, 1); mbar_init(p_bar + 8 * x, 4); mbar_init(p_bar + 16 + 8 * x, 4); mbar_init(o_bar + 8 * x, 1); }
        for (int x = 0; x < 2; ++x) { mbar_init(in_bar + 8 * x, 4); mbar_init(told_bar + 8 * x, 1); }
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
    release_dependents();                                  // not before the wait: ecco_paged_few_kernel relies on the order of the two
    const int32_t n_blocks = __ldcg(sc.n_blocks), total = n_blocks > 0 ? __ldcg(sc.block_tiles + n_blocks) : 0;
    const UnitSplit split(static_cast<int64_t>(total) * kv.heads, static_cast<int>(gridDim.x));
    const int64_t u0 = split.begin(static_cast<int>(blockIdx.x)), u1 = split.begin(static_cast<int>(blockIdx.x) + 1);
    const int32_t T = paged_tiles(kv);
    const bool causal = o.causal;
    // The whole warp waits; one vote decides, so that the branches are the warp's.  (A loop of each lane's own took 250 clocks to see a barrier
    // that had long been passed, this one 50.)  A wait that has run out makes all others run out at once.
    auto wait = [&](uint32_t bar, uint32_t parity) {
        constexpr unsigned full = 0xffffffffu;
        if (__all_sync(full, mbar_try_wait(bar, parity))) return true;
        for (int i = 0; i < 2 * kWaitLimit; ++i) {
            if (__all_sync(full, mbar_try_wait(bar, parity))) return true;
            if ((i & 63) == 63 && __any_sync(full, *failed)) break;
        }
        *failed = 1;
        atomicExch(&g_device_status, ECCO_ERR_DEVICE_TIMEOUT);
        return false;
    };

    // 384 threads x 168 registers = 128 x 40 + 256 x 232; 512 x 128 = 256 x 48 + 256 x 208
    if (k8) {
        if (warp >= 8) asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
        else asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    } else {
        if (warp >= 8) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        else asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
    }
    if (warp < 8) {
        // softmax: thread t of tile x holds row 128 x + t
        const uint32_t x = warp >> 2, t = threadIdx.x & 127u, s_at = tmem + ((warp & 3u) << 21) + x * 128, o_at = s_at + 256;
        const int32_t in_tile = static_cast<int32_t>(t) / o.q_per_kv, g = static_cast<int32_t>(t) - in_tile * o.q_per_kv;       // new token, query head
        // a scale of zero as a small one: times minus infinity it is still minus infinity
        const float scale = fabsf(o.scale_log2) < 1e-30f ? 1e-30f : o.scale_log2, unseen = scale > 0.0f ? -INFINITY : INFINITY;
        uint32_t n_piece = 0, n_s = 0, n_o = 0, n_join = 0;        // pieces, S, O and joins waited for
        bool ok = true;
        for (int64_t u = u0; u < u1 && ok;) {
            ok = wait(q_bar + 8 * x, n_piece & 1u);
            if (!ok) break;
            const ManyTask pc = tasks[(n_piece & 1u) * 2 + x];
            ++n_piece;
            warp_arrive(q_free + 8 * x);                   // the task has been read: with the products' arrival the next may come
            u += pc.to - pc.from;
            if (!pc.used) continue;
            const int32_t token = pc.token + in_tile;
            const bool exists = in_tile < tile_rows_tokens(o.q_per_kv) && token < pc.r_rows;
            const int64_t out_row = static_cast<int64_t>(pc.r_row0 + token) * o.q_heads + (kv.head0 + pc.head) * o.q_per_kv + g;
            const int32_t seen = exists ? tokens_seen(PagedReq{0, 0, pc.r_kv, 0, pc.r_rows, false}, token, causal) : 0;
            float m = -INFINITY, l = 0.0f;                 // m in units of log2, the weights stand at 2^(s - m + kManyWeightLog2)
            for (int32_t j = pc.from; j < pc.to; ++j) {
                ok = wait(s_bar + 8 * x, n_s++ & 1u);
                if (!ok) break;
                tmem_fence_after();
                float s[128];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(reinterpret_cast<uint32_t*>(s) + 32 * c, s_at + 32 * c);
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < 4; ++c) tie32(reinterpret_cast<uint32_t*>(s) + 32 * c);
                const int32_t left = seen - j * kManyTokens;           // columns that the row sees
                if (__any_sync(0xffffffffu, left < kManyTokens)) {
#pragma unroll
                    for (int c = 0; c < 128; ++c) s[c] = c < left ? s[c] : unseen;
                }
                float top;
                if (scale > 0.0f) {
                    float top4[4] = {fmaxf(s[0], s[1]), fmaxf(s[2], s[3]), fmaxf(s[4], s[5]), fmaxf(s[6], s[7])};
#pragma unroll
                    for (int c = 8; c < 128; c += 2) top4[(c >> 1) & 3] = max3(top4[(c >> 1) & 3], s[c], s[c + 1]);
                    top = fmaxf(max3(top4[0], top4[1], top4[2]), top4[3]) * scale;
                } else {
                    top = s[0];
#pragma unroll
                    for (int c = 1; c < 128; ++c) top = fminf(top, s[c]);
                    top *= scale;
                }
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
                            tie32(v);
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * f);
                            tmem_st32(o_at + 32 * c, v);
                        }
                    }
                }
                const float sub = kManyWeightLog2 - (m == -INFINITY ? 0.0f : m);
                // in two halves: the products of the first begin while the second is formed
                const uint64_t scale2 = pack_f2(scale, scale), sub2 = pack_f2(sub, sub);
                uint64_t sums[2] = {0, 0};                 // pairs of zeros
                uint32_t p[32];
                auto weights = [&](int from, int to) {
#pragma unroll
                    for (int c = from; c < to; ++c) {
                        float a, b;
                        unpack_f2(fma_f2(pack_f2(s[2 * c], s[2 * c + 1]), scale2, sub2), a, b);
                        a = exp2_fast(a);
                        b = exp2_fast(b);
                        sums[c & 1] = add_f2(sums[c & 1], pack_f2(a, b));
                        p[c & 31] = pack_h2(a, b);
                    }
                };
                auto sent = [&](int h) {
                    tmem_wait_st();
                    tmem_fence_before();
                    warp_arrive(p_bar + 16 * h + 8 * x);
                };
                weights(0, 32);
                tmem_st32(s_at, p);
                weights(32, 40);                           // while the first half is on its way
                sent(0);
                weights(40, 64);
                tmem_st32(s_at + 32, p);
                sent(1);
                float sum_a, sum_b;
                unpack_f2(add_f2(sums[0], sums[1]), sum_a, sum_b);
                l += sum_a + sum_b;
            }
            if (!ok) break;
            ok = wait(o_bar + 8 * x, n_o++ & 1u);
            if (!ok) break;
            tmem_fence_after();
            const bool whole = pc.whole;
            const float inv = inverse_of(l);
            // a piece's sums: 16 bytes of all rows of a tile side by side, so that the threads' stores, and the loads that join them, are whole lines
            auto sums_of = [&](int64_t slot) { return reinterpret_cast<float4*>(o.part + (slot * kManyRows + x * 128) * kGroup) + t; };
            {
                uint32_t v[128];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(v + 32 * c, o_at + 32 * c);
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < 4; ++c) tie32(v + 32 * c);
                if (exists && whole) {
                    uint4* const dst = reinterpret_cast<uint4*>(o.out + out_row * kGroup);
                    // a row that has seen nothing: O may not have been written at all
                    auto two = [&](int i) { return l != 0.0f ? pack_h2(__uint_as_float(v[i]) * inv, __uint_as_float(v[i + 1]) * inv) : 0u; };
#pragma unroll
                    for (int i = 0; i < 16; ++i) dst[i] = make_uint4(two(8 * i), two(8 * i + 2), two(8 * i + 4), two(8 * i + 6));
                } else if (exists) {
                    uint4* const dst = reinterpret_cast<uint4*>(sums_of(pc.slot));
#pragma unroll
                    for (int i = 0; i < 32; ++i) dst[i * 128] = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                }
                __syncwarp();
            }
            if (exists) {
                if (whole) { if (o.lse) o.lse[out_row] = lse_of(m, l, kManyWeightLog2); }
                else o.part_ml[static_cast<int64_t>(pc.slot) * kManyRows + x * 128 + t] = make_float2(m, l);
            }
            tmem_fence_before();                           // O has been read before the next block's P arrives
            if (!whole) {
                // The tile's four warps count themselves in; the last run's read all pieces.  (They meet at barriers whose
                // waits are bounded: a warp that has given up does not come.)
                __threadfence();
                warp_arrive(in_bar + 8 * x);
                if ((warp & 3u) == 0 && wait(in_bar + 8 * x, n_join & 1u)) {
                    if (lane == 0) last_in[x] = atomicAdd(sc.tickets + 2 * pc.run_lo + x, 1) == pc.run_hi - pc.run_lo;
                    warp_arrive(told_bar + 8 * x);
                }
                ok = wait(told_bar + 8 * x, n_join++ & 1u);
                if (!ok) break;
                if (last_in[x]) {
                    __threadfence();
                    // a thread to a row, 32 columns at a time: two pieces' loads are on their way together
#pragma unroll 1
                    for (int c = 0; c < 4 && exists; ++c) {
                        float jm = -INFINITY, jl = 0.0f;
                        float4 acc[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) acc[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 1
                        for (int w0 = pc.run_lo; w0 <= pc.run_hi; w0 += 2) {
                            float2 ml[2];
                            float4 v[2][8];
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                const int w = min(w0 + k, pc.run_hi);
                                const int64_t slot = 2 * static_cast<int64_t>(w) + (w == pc.run_lo ? pc.second : 0);
                                ml[k] = __ldcg(o.part_ml + slot * kManyRows + x * 128 + t);
#pragma unroll
                                for (int i = 0; i < 8; ++i) v[k][i] = __ldcg(sums_of(slot) + (8 * c + i) * 128);
                            }
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                if (w0 + k > pc.run_hi) break;
                                const float m0 = jm, l0 = jl;
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                    jm = m0;
                                    jl = l0;
                                    join_sums(jm, jl, acc[i], ml[k], v[k][i]);
                                }
                            }
                        }
                        const float j_inv = inverse_of(jl);
                        uint4* const dst = reinterpret_cast<uint4*>(o.out + out_row * kGroup) + 4 * c;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float4 a = acc[2 * i], b = acc[2 * i + 1];
                            dst[i] = make_uint4(pack_h2(a.x * j_inv, a.y * j_inv), pack_h2(a.z * j_inv, a.w * j_inv), pack_h2(b.x * j_inv, b.y * j_inv), pack_h2(b.z * j_inv, b.w * j_inv));
                        }
                        if (o.lse && c == 0) o.lse[out_row] = lse_of(jm, jl, kManyWeightLog2);
                    }
                }
            }
        }
    } else if (k8 && warp == 8) {
        // loads of E4M3 numbers, K and V by turns in the order in which they are used; a lane to a block of tokens that share a power of two.  The pages
        // of a tile are looked up with the tile before it.
        const int piece_shift = min(7, kv.page_shift), block_shift = min(4, kv.page_shift), n_scaled = 128 >> block_shift;
        const int32_t in_page = (1 << kv.page_shift) - 1;
        const int64_t n_scales = static_cast<int64_t>(kv.n_pages) * kv.all_heads << (kv.page_shift - block_shift);
        int32_t* const lefts = reinterpret_cast<int32_t*>(smem + 112);
        uint32_t n = 0;
        bool ok = true;
        for (int64_t u = u0; u < u1 && ok;) {
            const ManyPiece pc = many_piece(sc, kv.heads, n_blocks, total, u, u1);
            const PagedReq q = paged_req(kv, pc.r, T);
            u = pc.next;
            const int32_t head = kv.head0 + pc.head;
            auto page_of = [&](int32_t j, int i) {         // -1: none, -2: there is nothing to look for
                const int64_t token = static_cast<int64_t>(j) * kManyTokens + (i << block_shift), e = token >> kv.page_shift;
                if (j >= pc.to || i >= n_scaled || token >= q.kv) return -2;
                return e < kv.stride ? max(__ldcg(kv.tables + static_cast<int64_t>(pc.r) * kv.stride + e), -1) : -1;
            };
            int32_t page_next = page_of(pc.from, static_cast<int>(lane));
            for (int32_t j = pc.from; j < pc.to && ok; ++j) {
                const int32_t page_now = page_next;
                page_next = page_of(j + 1, static_cast<int>(lane));
                for (int which = 0; which < 2; ++which) {
                    const uint32_t st = n % kCodeStages, bar = code_at + 8 * st;
                    if (n >= kCodeStages) ok = wait(code_free + 8 * st, (n / kCodeStages - 1) & 1u);
                    if (!ok) break;
                    ++n;
                    for (int i = static_cast<int>(lane); i < n_scaled; i += 32) {
                        const int32_t page = i < 32 ? page_now : page_of(j, i), place = static_cast<int32_t>((static_cast<int64_t>(j) * kManyTokens + (i << block_shift)) & in_page);
                        const uint32_t words = base + ManyShape<k8>::kWords + st * 128 * 8 + i * 8;
                        if (page == -1 || page >= kv.n_pages) atomicExch(&g_device_status, ECCO_ERR_INVALID_ARG);
                        if (page < 0 || page >= kv.n_pages) {
                            sts_v2(words, 127u, 0u);
                            continue;
                        }
                        const int64_t of_head = static_cast<int64_t>(page) * kv.all_heads + head;
                        if (((i << block_shift) & ((1 << piece_shift) - 1)) == 0) {
                            const uint32_t to = base + ManyShape<k8>::kCodes + st * kCodeBytes + (i << (block_shift + 7)), bytes = 1u << (piece_shift + 7);
                            mbar_expect_more(bar, bytes);
                            if (kv.page_shift >= kP8SwizzledShift) tma_load_4d(to, which ? &v_map : &k_map, 0, place, head, page, bar);
                            else bulk_g2s(to, (which ? kv.v_blocks : kv.k_blocks) + ((of_head << kv.page_shift) + place) * kGroup, bytes, bar);
                        }
                        const int64_t scale = (of_head << (kv.page_shift - block_shift)) + (place >> block_shift), word = scale & ~3ll;
                        copy_word(words, (which ? kv.v_meta : kv.k_meta) + word, static_cast<int>(min(n_scales - word, static_cast<int64_t>(4))));
                        sts_u32(words + 4, static_cast<uint32_t>(scale & 3) * 8);
                    }
                    arrive_with_words(bar);
                    __syncwarp();
                    if (lane == 0) {                       // and what has been written here
                        lefts[st] = q.kv - j * kManyTokens;
                        mbar_arrive(bar);
                    }
                }
            }
        }
        if (!ok)                                           // what is on its way lands before the CTA leaves
            for (uint32_t i = n < kCodeStages ? 0 : n - kCodeStages; i < n; ++i)
                for (int k = 0; k < kWaitLimit && !mbar_try_wait(code_at + 8 * (i % kCodeStages), (i / kCodeStages) & 1u); ++k) {}
    } else if (k8 && warp >= 12) {
        // E4M3 numbers into operands: thread t has row t
        const uint32_t t = threadIdx.x - 384u, block_shift = static_cast<uint32_t>(min(4, kv.page_shift)), swizzle = kv.page_shift >= kP8SwizzledShift ? t & 7u : 0u;
        const uint32_t second = ((t >> 2) & 1u) << 4;      // the halves of a row's 32 bytes
        const volatile int32_t* const lefts = reinterpret_cast<const volatile int32_t*>(smem + 112);
        const int64_t n_all = 2 * (u1 - u0);
        for (int64_t i = 0; i < n_all; ++i) {
            const uint32_t n = static_cast<uint32_t>(i), cs = n % kCodeStages, st = n % kManyStages;
            if (!wait(code_at + 8 * cs, (n / kCodeStages) & 1u)) break;
            const uint32_t codes = base + ManyShape<k8>::kCodes + cs * kCodeBytes + t * kGroup, words = base + ManyShape<k8>::kWords + cs * 128 * 8 + (t >> block_shift) * 8;
            const uint32_t to = ring + st * kOperandBytes + t * 32;
            const int32_t left = lefts[cs];                // tokens that there are; behind them zeros, which any weight may meet
            const uint32_t by = power_h2(p8_exponent((lds_u32(words) >> lds_u32(words + 4)) & 0xffu));
            bool ok = true;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint4 x[4];
#pragma unroll
                for (int d = 0; d < 4; ++d) x[d] = lds_v4(codes + (((half * 4 + d) ^ swizzle) << 4));
                if (left < 128 && static_cast<int32_t>(t) >= left)
#pragma unroll
                    for (int d = 0; d < 4; ++d) x[d] = make_uint4(0u, 0u, 0u, 0u);
                if (half) warp_arrive(code_free + 8 * cs);                          // the numbers have been read
                else if (n >= kManyStages) ok = wait(free_at + 8 * st, (n / kManyStages - 1) & 1u);
                if (!ok) break;
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const uint32_t row = to + (half * 4 + d) * 4096;
                    sts_v4(row + second, mul_h2(e4m3_low(x[d].x), by), mul_h2(e4m3_high(x[d].x), by), mul_h2(e4m3_low(x[d].y), by), mul_h2(e4m3_high(x[d].y), by));
                    sts_v4(row + (second ^ 16u), mul_h2(e4m3_low(x[d].z), by), mul_h2(e4m3_high(x[d].z), by), mul_h2(e4m3_low(x[d].w), by), mul_h2(e4m3_high(x[d].w), by));
                }
            }
            if (!ok) break;
            fence_async_smem();                            // for the tensor cores to see
            warp_arrive(full_at + 8 * st);
        }
    } else if (!k8 && warp == 8) {
        // loads: K and V tiles in the order in which they are used
        uint32_t n = 0;
        bool ok = true;
        for (int64_t u = u0; u < u1 && ok;) {
            const ManyPiece pc = many_piece(sc, kv.heads, n_blocks, total, u, u1);
            const PagedReq q = paged_req(kv, pc.r, T);
            u = pc.next;
            for (int32_t j = pc.from; j < pc.to && ok; ++j) {
                for (int which = 0; which < 2; ++which) {
                    const uint32_t st = n % kManyStages, bar = full_at + 8 * st;
                    if (n >= kManyStages) ok = wait(free_at + 8 * st, (n / kManyStages - 1) & 1u);
                    if (!ok) break;
                    ++n;
                    if (lane == 0) {
                        mbar_expect_tx(bar, kOperandBytes);
                        // four tiles of 32 tokens, their pieces side by side; tiles that are not the request's are not used
                        tma_load_3d(ring + st * kOperandBytes, &k_map, 0, (which * kv.heads + pc.head) * kv.max_tiles + q.first + 4 * j, 0, bar);
                    }
                    __syncwarp();
                }
            }
        }
        if (!ok)                                           // what is on its way lands before the CTA leaves
            for (uint32_t i = n < kManyStages ? 0 : n - kManyStages; i < n; ++i)
                for (int k = 0; k < kWaitLimit && !mbar_try_wait(full_at + 8 * (i % kManyStages), (i / kManyStages) & 1u); ++k) {}
    } else if (warp == 9) {
        // products: of one tile of the rows while the other's softmax runs
        const uint32_t tmem_u = static_cast<uint32_t>(same_in_warp(static_cast<int>(tmem)));
        const uint64_t q_op = operand(q_smem, 16, 256), k_op = operand(ring, 16, 256), v_op = operand(ring, 4096, 256);
        constexpr uint64_t kStep = kOperandBytes >> 4;     // from one tile to the next, in an operand's units
        int n_q = 0, n_p[2] = {0, 0};                      // rows of Q and weights waited for
        int st = 0, turn = 0;                              // place in the ring, times around
        bool ok = true;
        auto advance = [&]() { if (++st == kManyStages) { st = 0; ++turn; } };
        for (int64_t u = u0; u < u1 && ok;) {
            ok = wait(q_bar, n_q & 1) && wait(q_bar + 8, n_q & 1) && wait(full_at + 8 * st, turn & 1);
            if (!ok) break;
            const ManyTask* const pc = tasks + (n_q & 1) * 2;
            ++n_q;
            const bool two = same_in_warp(pc[1].used) != 0;
            const int n_tiles = same_in_warp(pc->to - pc->from), steps_left = k8 ? INT_MAX : same_in_warp(max(pc->tiles - 4 * pc->from, 0) * 2);       // k8: no rows but the request's, or zeros
            u += n_tiles;
            tmem_fence_after();
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                if (x && !two) break;
                mma_scores(tmem_u + x * 128, q_op + x * kStep, k_op + st * kStep);
                mma_commit(s_bar + 8 * x);
            }
            if (n_tiles == 1) { mma_commit(q_free); mma_commit(q_free + 8); }
            mma_commit(free_at + 8 * st);
            advance();
            for (int j = 0; j < n_tiles && ok; ++j) {
                const int v_st = st, steps = k8 ? 8 : min(steps_left - 8 * j, 8);        // sixteen tokens at a time, as far as there are tiles
                const bool more = j + 1 < n_tiles;
                ok = wait(full_at + 8 * st, turn & 1);
                advance();
                if (ok && more) ok = wait(full_at + 8 * st, turn & 1);           // the next K tile: not to be waited for behind the products
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if (x && !two) break;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (ok) ok = wait(p_bar + 16 * h + 8 * x, n_p[x] & 1);
                        if (!ok) break;
                        tmem_fence_after();
                        const uint64_t v_half = v_op + v_st * kStep + h * 128;
                        if (steps == 8) mma_values4(tmem_u + 256 + x * 128, tmem_u + x * 128 + h * 32, v_half, j > 0 || h > 0);
                        else
#pragma unroll 1
                            for (int ks = 0; ks < min(4, steps - 4 * h); ++ks)
                                mma_values(tmem_u + 256 + x * 128, tmem_u + x * 128 + h * 32 + ks * 8, v_half + ks * 32, j > 0 || h > 0 || ks > 0);
                    }
                    if (!ok) break;
                    ++n_p[x];
                    if (more) {
                        mma_scores(tmem_u + x * 128, q_op + x * kStep, k_op + st * kStep);
                        mma_commit(s_bar + 8 * x);
                    } else {
                        mma_commit(o_bar + 8 * x);
                    }
                }
                if (!ok) break;
                mma_commit(free_at + 8 * v_st);
                if (more) { mma_commit(free_at + 8 * st); advance(); }
                if (j + 2 == n_tiles) { mma_commit(q_free); mma_commit(q_free + 8); }       // the piece's last scores are on their way
            }
        }
        if (!ok) {                                         // what has been issued ends before tensor memory is given back
            mma_commit(end_bar);
            for (int k = 0; k < kWaitLimit && !mbar_try_wait(end_bar, 0); ++k) {}
        }
    } else if (warp == 10) {
        // what there is to do, and the rows of Q: the next piece's while the last products of this one run
        const int32_t tokens = tile_rows_tokens(o.q_per_kv);
        uint32_t n = 0;
        for (int64_t u = u0; u < u1;) {
            const ManyPiece pc = many_piece(sc, kv.heads, n_blocks, total, u, u1);
            const PagedReq q = paged_req(kv, pc.r, T);
            const int64_t first = u - pc.from;             // the block's first unit
            const int run_lo = split.owner(first), run_hi = split.owner(first + pc.tiles - 1);
            if (n && !(wait(q_free, (n - 1) & 1u) && wait(q_free + 8, (n - 1) & 1u))) break;
            if (lane < 2) {                                // a lane to a tile of rows
                const uint32_t x = lane, bar = q_bar + 8 * x;
                const int32_t token = (2 * pc.block + static_cast<int32_t>(x)) * tokens;
                const bool used = token < q.rows;
                tasks[(n & 1u) * 2 + x] = ManyTask{used, pc.from, pc.to, q.tiles, pc.head, q.row0, q.rows, q.kv, token, pc.from == 0 && pc.to == pc.tiles,
                                                   2 * static_cast<int>(blockIdx.x) + (u == u0 ? 0 : 1), run_lo, run_hi, split.begin(run_lo) != first};
                mbar_expect_tx(bar, used ? 8 * 32 * tokens * o.q_per_kv : 0);
                if (used)
                    for (int d = 0; d < 8; ++d)
                        tma_load_3d(q_smem + x * kOperandBytes + d * 4096, &q_map, 16 * d, (kv.head0 + pc.head) * o.q_per_kv, q.row0 + token, bar);
            }
            __syncwarp();
            ++n;
            u = pc.next;
        }
        if (n && *failed)                                  // what is on its way lands before the CTA leaves
            for (uint32_t x = 0; x < 2; ++x)
                for (int k = 0; k < kWaitLimit && !mbar_try_wait(q_bar + 8 * x, (n - 1) & 1u); ++k) {}
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

}  // namespace
