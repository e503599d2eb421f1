// ecco_paged_kernels.cuh -- K6: the paged KV cache: slots and block tables, pages into tiles, attention of few rows
// Part of the one translation unit ecco_kernels.cu; included from there only.
#pragma once

namespace {

// ---------------------------------------------------------------------------------------------
// K6p: block tables and slots from request lengths.  One launch; every CTA forms the prefix sums of all requests itself (8 bytes a
// request, which stay in L2) and writes the rows of d_slots that are its share: no CTA waits for another.
// Requests pass in rounds of kPlanThreads; a round's prefix sums lie in shared memory, and a row finds its request there by bisection.
// A page is appended to its table by the row that holds the page's first token, which is always a new one.
// ---------------------------------------------------------------------------------------------
constexpr int kPlanThreads = 1024;

struct PagedPlan {
    const int32_t *ctx, *added, *free_pages;
    int32_t *tables, *slots, *cu_new, *kv_lens, *kv_tiles, *result;
    int32_t page_shift, n_pages, n_req, n_free, stride, n_slots;
};

// inclusive prefix sums over the CTA of three numbers per thread; total: over all threads
struct Sum3 { int32_t a, b, c; };
__device__ __forceinline__ Sum3 scan3(Sum3 v, Sum3& total, Sum3 (&warp_sums)[32])
{
    constexpr unsigned full = 0xffffffffu;
    const int lane = static_cast<int>(threadIdx.x & 31u), warp = static_cast<int>(threadIdx.x >> 5);
    auto scan_warp = [&](Sum3& x) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t a = __shfl_up_sync(full, x.a, o), b = __shfl_up_sync(full, x.b, o), c = __shfl_up_sync(full, x.c, o);
            if (lane >= o) { x.a += a; x.b += b; x.c += c; }
        }
    };
    scan_warp(v);
    __syncthreads();                                       // the sums of the previous call have been read
    if (lane == 31) warp_sums[warp] = v;
    __syncthreads();
    Sum3 w = warp_sums[lane];
    scan_warp(w);
    total = {__shfl_sync(full, w.a, 31), __shfl_sync(full, w.b, 31), __shfl_sync(full, w.c, 31)};
    const int from = warp > 0 ? warp - 1 : 0;
    const int32_t a = __shfl_sync(full, w.a, from), b = __shfl_sync(full, w.b, from), c = __shfl_sync(full, w.c, from);
    if (warp > 0) { v.a += a; v.b += b; v.c += c; }
    return v;
}

__global__ void __launch_bounds__(kPlanThreads, 1)
ecco_paged_plan_kernel(const PagedPlan p)
{
    __shared__ Sum3 warp_sums[32];
    __shared__ long long totals[3];                        // new tokens, pages, tiles of all requests
    __shared__ int32_t first_row[kPlanThreads + 1], ctx_s[kPlanThreads], page_from[kPlanThreads];
    const int tid = static_cast<int>(threadIdx.x), lane = tid & 31;
    const int32_t page_size = 1 << p.page_shift;
    release_dependents();
    if (tid < 3) totals[tid] = 0;
    __syncthreads();
    dependency_wait();
    // lengths of request r; those behind the last are zero
    auto lengths = [&](int r, int32_t& ctx, int32_t& added) {
        ctx = r < p.n_req ? __ldcg(p.ctx + r) : 0;
        added = r < p.n_req ? __ldcg(p.added + r) : 0;
    };
    // first the totals: all requests are served or none
    bool fine = true;
    long long sum[3] = {0, 0, 0};
    int32_t ctx0 = 0, added0 = 0;                          // of the first round, which usually is the only one
    for (int r = tid; r < p.n_req; r += kPlanThreads) {
        int32_t ctx, added;
        lengths(r, ctx, added);
        if (r == tid) { ctx0 = ctx; added0 = added; }
        const long long kv = static_cast<long long>(ctx) + added;
        fine = fine && ctx >= 0 && added >= 0 && kv <= INT32_MAX && kv <= static_cast<long long>(p.stride) << p.page_shift;
        sum[0] += added;
        sum[1] += ((kv + page_size - 1) >> p.page_shift) - ((static_cast<long long>(ctx) + page_size - 1) >> p.page_shift);
        sum[2] += (kv + 31) >> 5;
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) {
#pragma unroll
        for (int o = 16; o; o >>= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
        if (lane == 0 && sum[i]) atomicAdd(reinterpret_cast<unsigned long long*>(&totals[i]), static_cast<unsigned long long>(sum[i]));
    }
    fine = __syncthreads_and(fine) && totals[0] <= INT32_MAX && totals[2] <= INT32_MAX;
    const int32_t status = !fine ? ECCO_ERR_INVALID_ARG : totals[0] > p.n_slots || totals[1] > p.n_free ? ECCO_ERR_WORKSPACE : 0;
    const int32_t n_new = status ? 0 : static_cast<int32_t>(totals[0]);
    if (blockIdx.x == 0 && tid < 4) p.result[tid] = tid == 0 ? status : status ? 0 : static_cast<int32_t>(totals[tid == 1 ? 1 : tid == 2 ? 0 : 2]);

    // this CTA's rows
    const int32_t per = static_cast<int32_t>((static_cast<long long>(p.n_slots) + gridDim.x - 1) / gridDim.x);
    const int32_t row0 = static_cast<int32_t>(min(static_cast<long long>(p.n_slots), static_cast<long long>(per) * blockIdx.x));
    const int32_t row1 = static_cast<int32_t>(min(static_cast<long long>(p.n_slots), static_cast<long long>(row0) + per));
    for (long long i = max(row0, n_new) + static_cast<long long>(tid); i < row1; i += kPlanThreads) p.slots[i] = -1;
    Sum3 before = {0, 0, 0};
    const int rounds = (p.n_req + kPlanThreads - 1) / kPlanThreads;
    for (int round = 0; round < rounds; ++round) {
        const int r = round * kPlanThreads + tid;
        int32_t ctx = ctx0, added = added0;
        if (round > 0) lengths(r, ctx, added);
        if (status) ctx = added = 0;
        const long long kv = static_cast<long long>(ctx) + added;
        const int32_t held = static_cast<int32_t>((static_cast<long long>(ctx) + page_size - 1) >> p.page_shift);
        const Sum3 mine = {added, static_cast<int32_t>((kv + page_size - 1) >> p.page_shift) - held, static_cast<int32_t>((kv + 31) >> 5)};
        Sum3 total;
        const Sum3 upto = scan3(mine, total, warp_sums);   // its barriers: the previous round's rows are done, see below
        first_row[tid] = before.a + upto.a - mine.a;
        ctx_s[tid] = ctx;
        page_from[tid] = before.b + upto.b - mine.b - held;      // free page of table entry e: page_from + e
        if (tid == 0) first_row[kPlanThreads] = before.a + total.a;
        if (static_cast<int>(blockIdx.x) == round % static_cast<int>(gridDim.x) && r < p.n_req) {
            p.kv_lens[r] = static_cast<int32_t>(kv);
            p.cu_new[r + 1] = before.a + upto.a;
            p.kv_tiles[r + 1] = before.c + upto.c;
        }
        __syncthreads();
        const int32_t from = max(row0, before.a), to = min(row1, before.a + total.a);
        for (long long row = from + static_cast<long long>(tid); row < to; row += kPlanThreads) {
            int lo = 0, hi = kPlanThreads;                 // the last request that begins at or before the row has it: empty ones begin before it
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (first_row[mid] <= row) lo = mid; else hi = mid;
            }
            const int32_t t = ctx_s[lo] + static_cast<int32_t>(row) - first_row[lo], e = t >> p.page_shift;
            int32_t* const entry = p.tables + static_cast<int64_t>(round * kPlanThreads + lo) * p.stride + e;
            const bool taken = e < (static_cast<int32_t>((static_cast<long long>(ctx_s[lo]) + page_size - 1) >> p.page_shift));
            const int32_t page = taken ? __ldcg(entry) : __ldcg(p.free_pages + page_from[lo] + e);
            if (!taken && (t & (page_size - 1)) == 0) *entry = page;
            p.slots[row] = page >= 0 && page < p.n_pages ? (page << p.page_shift) + (t & (page_size - 1)) : -1;
        }
        __syncthreads();
        before.a += total.a;
        before.b += total.b;
        before.c += total.c;
    }
    if (blockIdx.x == 0 && tid == 0) { p.cu_new[0] = 0; p.kv_tiles[0] = 0; }
}

// ---------------------------------------------------------------------------------------------
// Attention over the pages.  The blocks are decoded once per call, by the decoder of ecco_decompress at its full rate, into
// tiles of 32 tokens in the workspace; the attention kernels read these.  A tile is 8 KB:
//   eight [32 tokens][16 dims] fp16 pieces of 1 KB, the 16-byte halves of a 32-byte row swapped in every second block of four rows
// which is what the decoder's staging pieces look like in shared memory, what ldmatrix reads without conflicts, and, for tcgen05, the
// canonical layout of both a K operand (contraction over dims, K-major) and a V operand (contraction over tokens, MN-major)
// with 32-byte swizzle.  One layout for all, moved by bulk copies.
// Decoding inside of the attention kernel instead leaves the decoder 17 warps (9.6 KB of tiles per warp and two sets of tables) instead
// of 31 and one symbol per lookup instead of two, and decodes again for every row tile.
// ---------------------------------------------------------------------------------------------
constexpr uint32_t kPieceBytes = 1024;                     // 32 tokens x 16 dims
constexpr uint32_t kKvTileBytes = 8 * kPieceBytes;

struct PagedKv {
    const uint8_t *k_meta, *v_meta, *k_blocks, *v_blocks;
    const int32_t *tables, *cu_new, *kv_lens, *kv_tiles;
    int32_t n_pages, page_shift, all_heads, stride, n_req, n_tokens, max_new, max_kv, max_tiles;
    int32_t head0, heads;      // KV heads of this launch
    uint8_t* staged;           // [K, V][heads][max_tiles] tiles
};
__device__ __forceinline__ uint8_t* staged_tile(const PagedKv& kv, int which, int head, int tile)
{
    return kv.staged + ((static_cast<uint64_t>(which) * kv.heads + head) * kv.max_tiles + tile) * kKvTileBytes;
}
// tiles of all requests, cut to what the workspace was made for
__device__ __forceinline__ int32_t paged_tiles(const PagedKv& kv) { return min(max(__ldcg(kv.kv_tiles + kv.n_req), 0), kv.max_tiles); }

// Where a request's tiles and rows are, whatever the arrays hold: inside of the workspace and of q.  cut: the arrays say something else, which
// paged_schedule reports (with fewer rows than the request has, for one, the causal mask of those that are left would be another one).
struct PagedReq { int32_t first, tiles, kv, row0, rows; bool cut; };
__device__ __forceinline__ PagedReq paged_req(const PagedKv& kv, int r, int32_t T)
{
    PagedReq q;
    const int32_t t0 = __ldcg(kv.kv_tiles + r), t1 = __ldcg(kv.kv_tiles + r + 1), c0 = __ldcg(kv.cu_new + r), c1 = __ldcg(kv.cu_new + r + 1), len = __ldcg(kv.kv_lens + r);
    q.first = min(max(t0, 0), T);
    q.tiles = min(max(t1, q.first), T) - q.first;
    q.kv = static_cast<int32_t>(min(static_cast<int64_t>(min(max(len, 0), kv.max_kv)), static_cast<int64_t>(q.tiles) * 32));
    q.row0 = min(max(c0, 0), kv.n_tokens);
    q.rows = min(max(c1, q.row0), kv.n_tokens) - q.row0;
    q.cut = q.first != t0 || q.first + q.tiles != t1 || q.kv != len || q.row0 != c0 || q.row0 + q.rows != c1;
    return q;
}
// The last r in 0 .. n - 1 with begin[r] <= x (0 if there is none), by the whole warp: 32 probes at a time.
__device__ __forceinline__ int warp_find(const int32_t* begin, int n, int32_t x)
{
    const int lane = static_cast<int>(threadIdx.x & 31u);
    int lo = 0;
    while (n > 1) {
        const int step = (n + 31) >> 5, at = lane * step;
        const bool below = at < n && __ldcg(begin + lo + at) <= x;
        const int last = max(31 - __clz(__ballot_sync(0xffffffffu, below)), 0);
        lo += last * step;
        n = min(step, n - last * step);
    }
    return lo;
}

constexpr int kManyRows = 256;                             // rows of a block of ecco_paged_many_kernel: two tiles of 128, as many whole tokens as these hold
constexpr int kManyTokens = 128;                           // tokens of its tiles of K and V
__host__ __device__ constexpr int32_t tile_rows_tokens(int32_t q_per_kv) { return 128 / q_per_kv; }      // new tokens of a tile of rows
// What the attention kernels need to know of a batch, made by paged_schedule.
struct PagedSchedule {
    int32_t* few_tiles;        // [n_req + 1]: prefix sums of the tiles of the requests for ecco_paged_few_kernel, at most all tiles that there are
    int32_t* block_tiles;      // [max_blocks + 1]: prefix sums of the 128-token tiles of all blocks
    int2* blocks;              // [max_blocks]: request, block of the request
    int32_t* n_blocks;
    int32_t* n_cuts;           // set to zero
    int32_t max_blocks, few_rows;
    int32_t* tickets;          // [n_tickets]: zero when ecco_paged_many_kernel begins
    int32_t n_tickets;
};

// A row of a request that begins in a run and goes on in the next ones, as ecco_paged_join_kernel needs it: its row of out, the place of the first
// piece's sums (slot * kFewRows + row), the runs of the first and of the last piece.
struct alignas(16) FewCut { int32_t out_row, place, first_run, last_run; };
struct PagedOut {
    const __half* q;
    int64_t q_stride;
    float scale_log2;          // scale * log2(e)
    int32_t q_per_kv, q_heads, causal;
    __half* out;
    float* lse;                // or NULL
    float* part;               // partial sums [slot][rows][128]
    float2* part_ml;           // maxima (log2) and sums of weights [slot][rows]
    FewCut* cuts;              // rows of cut requests, in any order
    int32_t* n_cuts;           // zero when ecco_paged_few_kernel begins
    int32_t discard;           // the tiles begin at multiples of 128 bytes
    const float* scores;       // [heads][max_tiles][score_rows][32]: products of q and K, see K6k
    int32_t score_rows;
    int32_t early;             // ecco_paged_few_kernel comes behind ecco_paged_many_kernel
};
// tokens that row i of a request sees
__device__ __forceinline__ int32_t tokens_seen(const PagedReq& q, int32_t token, bool causal)
{
    return causal ? min(max(q.kv - q.rows + token + 1, 0), q.kv) : q.kv;
}
// tokens that the rows of a block see together: those of its last row
__device__ __forceinline__ int32_t block_sees(const PagedReq& q, int32_t block, int32_t q_per_kv, bool causal)
{
    return tokens_seen(q, min((block + 1) * 2 * tile_rows_tokens(q_per_kv), q.rows) - 1, causal);
}
// By one warp: which requests are for which kernel, and the two lines of tiles.  A block that sees nothing counts as one tile, so that
// somebody writes its rows.
__device__ __forceinline__ void paged_schedule(const PagedKv& kv, const PagedSchedule& sc, const PagedOut& o)
{
    const int32_t q_per_kv = o.q_per_kv;
    constexpr unsigned full = 0xffffffffu;
    const int lane = static_cast<int>(threadIdx.x & 31u);
    const int32_t T = paged_tiles(kv);
    auto scan = [&](int32_t v) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t x = __shfl_up_sync(full, v, o);
            if (lane >= o) v += x;
        }
        return v;
    };
    int32_t few = 0, tiles = 0, n_blocks = 0;
    if (lane == 0) { sc.few_tiles[0] = 0; sc.block_tiles[0] = 0; *sc.n_cuts = 0; }
    for (int i = lane; i < sc.n_tickets; i += 32) sc.tickets[i] = 0;
    PagedReq next = {};
    if (lane < kv.n_req) next = paged_req(kv, lane, T);
    for (int r0 = 0; r0 < kv.n_req; r0 += 32) {
        const int r = r0 + lane;
        const PagedReq q = next;
        next = {};
        if (r + 32 < kv.n_req) next = paged_req(kv, r + 32, T);        // on their way while these are dealt with
        const int64_t rows = static_cast<int64_t>(q.rows) * q_per_kv;
        if (r < kv.n_req && (q.rows > kv.max_new || q.cut)) atomicExch(&g_device_status, ECCO_ERR_INVALID_ARG);
        const bool many = rows > sc.few_rows;
        // Requests that share no tile have T together at most.  Prefix sums that go up and down could give any number: beyond T there is
        // nothing, so that no place in the line passes 32 bits.  (Such a request is cut, and reported; 32 times T is below 2^31.)
        const int32_t f = static_cast<int32_t>(min(static_cast<int64_t>(few) + scan(!many && rows > 0 ? q.tiles : 0), static_cast<int64_t>(T)));
        if (r < kv.n_req) sc.few_tiles[r + 1] = f;
        few = __shfl_sync(full, f, 31);
        // requests without a token: nobody else comes to their rows
        for (unsigned left = __ballot_sync(full, !many && rows > 0 && q.tiles == 0); left; left &= left - 1u) {
            const int src = __ffs(left) - 1;
            const int64_t row0 = __shfl_sync(full, q.row0, src), heads = kv.heads * q_per_kv, n = __shfl_sync(full, q.rows, src) * heads;
            for (int64_t i = 0; i < n; ++i) {
                const int64_t at = (row0 + i / heads) * o.q_heads + kv.head0 * q_per_kv + i % heads;
                reinterpret_cast<uint2*>(o.out + at * kGroup)[lane] = make_uint2(0u, 0u);
                if (o.lse && lane == 0) o.lse[at] = -INFINITY;
            }
        }
        for (unsigned left = __ballot_sync(full, many); left; left &= left - 1u) {
            const int src = __ffs(left) - 1;
            PagedReq one;
            one.rows = __shfl_sync(full, q.rows, src);
            one.kv = __shfl_sync(full, q.kv, src);
            const int32_t per_block = 2 * tile_rows_tokens(q_per_kv), blocks = (one.rows + per_block - 1) / per_block;
            for (int32_t b0 = 0; b0 < blocks && n_blocks < sc.max_blocks; b0 += 32) {
                const int32_t b = b0 + lane, n = min(min(blocks - b0, 32), sc.max_blocks - n_blocks);
                const int32_t mine = lane < n ? max((block_sees(one, b, q_per_kv, o.causal) + kManyTokens - 1) / kManyTokens, 1) : 0;
                const int32_t upto = tiles + scan(mine);
                if (lane < n) {
                    sc.blocks[n_blocks + lane] = make_int2(r0 + src, b);
                    sc.block_tiles[n_blocks + lane + 1] = upto;
                }
                tiles = __shfl_sync(full, upto, 31);
                n_blocks += n;
            }
        }
    }
    if (lane == 0) *sc.n_blocks = n_blocks;
}

// The request that a tile belongs to, and the tile's first token in it: from the prefix sums in the misc area (`firsts`) or, of more requests
// than find room there, in memory.
constexpr int kStageTiles = 224;
__device__ __forceinline__ void fetch_firsts(const PagedKv& kv, int32_t* firsts)
{
    if (kv.n_req <= kStageTiles)
        for (int i = static_cast<int>(threadIdx.x); i <= kv.n_req; i += static_cast<int>(blockDim.x)) firsts[i] = __ldcg(kv.kv_tiles + i);
    __syncthreads();
}
__device__ __forceinline__ int request_of(const PagedKv& kv, const int32_t* firsts, int32_t tile, int32_t& first)
{
    int r = 0;
    if (kv.n_req <= kStageTiles) {                         // the last request that begins at or before the tile
        for (int n = kv.n_req; n > 1;) {
            const int half = n >> 1;
            if (firsts[r + half] <= tile) { r += half; n -= half; } else n = half;
        }
        first = firsts[r];
    } else {
        r = warp_find(kv.kv_tiles, kv.n_req, tile);
        first = __ldcg(kv.kv_tiles + r);
    }
    return r;
}
// The block of a request's token for a KV head of the launch, NULL where there is none.
__device__ __forceinline__ const uint8_t* paged_block(const PagedKv& kv, const uint8_t* blocks, int r, int64_t token, int32_t head)
{
    const int64_t e = token >> kv.page_shift;
    const int32_t len = __ldcg(kv.kv_lens + r), page = e >= 0 && e < kv.stride ? __ldcg(kv.tables + static_cast<int64_t>(r) * kv.stride + e) : -1;
    if (token < 0 || token >= len) return nullptr;
    if (page < 0 || page >= kv.n_pages) {
        atomicExch(&g_device_status, ECCO_ERR_INVALID_ARG);
        return nullptr;
    }
    const int64_t at = ((static_cast<int64_t>(page) * kv.all_heads + kv.head0 + head) << kv.page_shift) + (token & ((1 << kv.page_shift) - 1));
    return blocks + at * kBlockBytes;
}

// K6s: pages -> tiles.  ecco_decompress_tma_kernel with another way in (a lane finds its token's block through the request's table)
// and out (a piece leaves by one bulk copy of 1 KB).
//   kHalves: even CTAs decode K, odd ones V: no CTA needs both sets of tables, and small calls decode K and V side by side.
//   kBoth: every CTA decodes its share of K, then of V: another 4 us for the second set of tables, but caches
//   whose blocks take differently long leave no CTA waiting (2.1 M groups of K and of V, 178 and 146 us by ecco_decompress: 377 -> 362 us).
// Values are clamped to fp16's finite range (once per group, on the sixteen values of its table): weight zero times an infinity would
// be NaN in rows that do not see the token.
//   kOnlyV: V alone, see ecco_paged_scores_kernel.
enum StageKind { kHalves, kBoth, kOnlyV };
template <int kMaxWarps, StageKind kKind>
__global__ void __launch_bounds__(kMaxWarps * 32, 1)
ecco_paged_stage_kernel(const __grid_constant__ PagedKv kv, const __grid_constant__ PagedOut o, const __grid_constant__ PagedSchedule sc)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint32_t cta = kKind == kHalves ? blockIdx.x >> 1 : blockIdx.x, ctas = kKind == kHalves ? gridDim.x >> 1 : gridDim.x;
    const uint32_t swz = ((lane >> 2) & 1u) << 4;
    int32_t* const firsts = reinterpret_cast<int32_t*>(smem + 64);
    static_assert(64 + (kStageTiles + 1) * 4 <= kMisc, "the prefix sums fit the misc area");
    release_dependents();
    for (int phase = 0; phase < (kKind == kBoth ? 2 : 1); ++phase) {
        const int which = kKind == kBoth ? phase : kKind == kOnlyV ? 1 : static_cast<int>(blockIdx.x & 1u);
        const uint8_t* const d_meta = which ? kv.v_meta : kv.k_meta;
        const DecodeTables tb = plan_decode_tables(smem_u32(smem), d_meta, true);
        if (phase) {                                       // see ecco_decompress_tma_kernel
            fence_async_smem();
            __syncthreads();
        }
        issue_decode_tables(tb, d_meta, phase == 0);
        const uint32_t tiles_base = (tb.warp_base + 1023u) & ~1023u;
        const uint32_t nw = decode_warps(tb, kTmaWarpBytes, tiles_base - tb.warp_base);
        const uint32_t stage = tiles_base + warp * 1024;
        const uint32_t bits = tiles_base + nw * 1024 + warp * kBitBytes + lane * 4;
        const uint32_t my_row = stage + lane * 32;
        const bool ready = finish_decode_tables(tb, static_cast<uint32_t>(phase));
        if (phase == 0) {                                  // without tables too: the next kernels rely on the schedule
            dependency_wait();
            fetch_firsts(kv, firsts);
            // one warp, if possible one that has no room to decode, makes the schedule on the side
            if (blockIdx.x == 0 && warp == (nw < blockDim.x >> 5 ? nw : 0u)) paged_schedule(kv, sc, o);
            if (blockIdx.x == 0 && threadIdx.x == 0 && __ldcg(kv.kv_tiles + kv.n_req) > kv.max_tiles) atomicExch(&g_device_status, ECCO_ERR_INVALID_ARG);
        }
        if (!ready) return;
        const float T = tb.T;
        const uint32_t n_tiles = static_cast<uint32_t>(paged_tiles(kv)), units = n_tiles * kv.heads;
        const uint32_t tile_stride = balanced_warps(units, ctas * nw);
        uint32_t u = warp * ctas + cta;
        if (warp >= nw || u >= tile_stride) u = units;

        const uint8_t* const blocks = which ? kv.v_blocks : kv.k_blocks;
        auto block_ptr = [&](uint32_t unit) {
            const uint32_t head = unit / n_tiles;
            const int32_t tile = static_cast<int32_t>(unit - head * n_tiles);
            int32_t first;
            const int r = request_of(kv, firsts, tile, first);
            return paged_block(kv, blocks, r, (static_cast<int64_t>(tile) - first) * 32 + lane, static_cast<int32_t>(head));
        };
        const uint8_t* next = u < units ? block_ptr(u) : nullptr;
        while (u < units) {
            const uint32_t head = u / n_tiles;
            uint8_t* const dst = staged_tile(kv, kKind == kOnlyV ? 0 : which, static_cast<int>(head), static_cast<int>(u - head * n_tiles));
            Block blk;
            const bool there = next != nullptr;
            if (there) {
                ldg_block(blk, next);
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) blk.w[i] = 0;     // whatever it decodes to: finite, and a token that no row sees
            }
            LaneGroup lg = open_block<true>(blk, bits, tb, T);
            u += tile_stride;
            if (u < units) {
                next = block_ptr(u);
                if (next) prefetch_block_l2(next);
            }
            auto send_piece = [&](int piece) {
                fence_async_smem();                            // generic-proxy writes -> visible to the engine
                __syncwarp();
                if (lane == 0) { bulk_s2g(dst + piece * kPieceBytes, stage, kPieceBytes); bulk_commit(); }
            };
            const uint32_t end = decode_group<kBlockBits, kBlockFreeSteps>(lg, bits, tb.pairs, [&](int i, uint32_t ranks, bool cutting, int n_ok) {
                uint32_t v[4];
                map_ranks(lg, ranks, v);
                if (cutting) cut_values(v, n_ok);
                if (!(i & 1)) {
                    if (lane == 0) bulk_wait_read0();          // the engine has read the previous piece
                    __syncwarp();
                    sts_v4(my_row + swz, v[0], v[1], v[2], v[3]);
                } else {
                    sts_v4(my_row + (swz ^ 16u), v[0], v[1], v[2], v[3]);
                    if (i != 15) send_piece(i >> 1);
                }
            });
            const int n_pad = pads_of(end);
            const int n_max = __reduce_max_sync(0xffffffffu, n_pad);
            if (n_max > 0) {
                if (lane == 0) bulk_wait_all();                // pieces 0..6 of this tile are in memory
                __syncwarp();
#pragma unroll 1
                for (int j = 0; j < n_max; ++j) {              // ascending: a later pad overrides an earlier one
                    if (j < n_pad) {
                        const uint32_t f = pad_field(bits, j), loc = f & 127u, byte = ((loc & 15u) * 2) ^ swz;
                        const float v = fminf(fmaxf(fp8_to_float(f >> 7) * T, -65504.0f), 65504.0f);
                        if (loc >= 112u) sts_u16(my_row + byte, f2h_bits(v));
                        else *reinterpret_cast<uint16_t*>(dst + (loc >> 4) * kPieceBytes + lane * 32 + byte) = static_cast<uint16_t>(f2h_bits(v));
                    }
                }
            }
            send_piece(7);
        }
        if (lane == 0) bulk_wait_all();                        // the staging piece may lie elsewhere in the next phase
    }
}

// K6k: products of K with one to eight rows of q per request (new tokens x query heads per KV head), instead of K in tiles:
// ecco_attn_scores_kernel and ecco_attn_scores_mma_kernel with another way to the blocks.  Half of the tiles need neither be written nor read.
// One or two rows are as fast as decoding K is (8 requests of 4048 tokens, 32 heads: 261 -> 223 us).  Three to eight go through the warp's
// own tiles to the tensor cores, with 20 warps and one symbol per lookup: slower than the decoder alone, but by less than K's way through
// memory takes (32 requests of 1 to 16384 tokens, 8 heads, three / eight rows: 530 / 531 -> 506 / 520 us).
//
// The walk over a warp's tiles: tile by tile of head by head; use(block, there, head, tile, request, whether the request or the head is another one)
template <class Use>
__device__ __forceinline__ void walk_tiles(const PagedKv& kv, const int32_t* firsts, int nw, Use&& use)
{
    const int lane = static_cast<int>(threadIdx.x & 31u), warp = static_cast<int>(threadIdx.x >> 5);
    const int32_t n_tiles = paged_tiles(kv);
    const int64_t U = static_cast<int64_t>(n_tiles) * kv.heads;
    const int wg = warp < nw ? warp * static_cast<int>(gridDim.x) + static_cast<int>(blockIdx.x) : INT_MAX;
    const int W = static_cast<int>(balanced_warps(static_cast<uint64_t>(U), gridDim.x * static_cast<uint32_t>(nw)));
    if (wg >= W) return;
    const UnitSplit split(U, W);
    const int64_t u0 = split.begin(wg);
    int32_t head = static_cast<int32_t>(divide(static_cast<uint64_t>(u0), static_cast<uint64_t>(n_tiles))), tile = static_cast<int32_t>(u0 - static_cast<int64_t>(head) * n_tiles);
    int32_t first;
    int r = request_of(kv, firsts, tile, first), of_head = -1, of_request = -1;
    auto block_ptr = [&]() { return paged_block(kv, kv.k_blocks, r, (static_cast<int64_t>(tile) - first) * 32 + lane, head); };
    const uint8_t* next = block_ptr();
    for (int left = static_cast<int>(split.begin(wg + 1) - u0); left > 0; --left) {
        const int32_t this_head = head, this_tile = tile;
        const int this_r = r;
        Block cur;
        const bool there = next != nullptr;
        if (there) {
            ldg_block(cur, next);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) cur.w[i] = 0;
        }
        if (left > 1) {
            if (++tile == n_tiles) { tile = 0; ++head; }
            r = request_of(kv, firsts, tile, first);
            next = block_ptr();
            if (next) prefetch_block_l2(next);
        }
        use(cur, there, this_head, this_tile, this_r, this_head != of_head || this_r != of_request);
        of_head = this_head;
        of_request = this_r;
    }
}
// Row i of a request's q for a head of the launch, NULL where there is none.
__device__ __forceinline__ const __half* paged_row(const PagedKv& kv, const PagedOut& o, const PagedReq& q, int32_t head, int i)
{
    const int token = i / o.q_per_kv, g = i - token * o.q_per_kv;
    return token < q.rows ? o.q + (q.row0 + token) * o.q_stride + (static_cast<int64_t>(kv.head0 + head) * o.q_per_kv + g) * kGroup : nullptr;
}
template <int kV, int kMaxWarps>
__global__ void __launch_bounds__(kMaxWarps * 32, 1)
ecco_paged_scores_kernel(const __grid_constant__ PagedKv kv, const __grid_constant__ PagedOut o, float* __restrict__ d_scores)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    int32_t* const firsts = reinterpret_cast<int32_t*>(smem + 64);
    release_dependents();
    const DecodeTables tb = plan_decode_tables(smem_u32(smem), kv.k_meta, true);
    const int nw = static_cast<int>(decode_warps(tb, scalar_warp_bytes(kV)));
    const int lane = static_cast<int>(threadIdx.x & 31u), warp = static_cast<int>(threadIdx.x >> 5);
    const uint32_t xs = tb.warp_base + warp * scalar_warp_bytes(kV);             // this warp's rows of q [kV][128] fp16
    const uint32_t bits = xs + kV * kGroup * 2 + kRankRows * 128 + lane * 4;
    issue_decode_tables(tb, kv.k_meta);
    if (!finish_decode_tables(tb)) return;
    dependency_wait();
    fetch_firsts(kv, firsts);
    const float T = tb.T;
    walk_tiles(kv, firsts, nw, [&](const Block& cur, bool there, int32_t head, int32_t tile, int r, bool other) {
        if (other) {
            // lane l brings elements 4l .. 4l+3 of every row; rows that there are not are zero
            const PagedReq q = paged_req(kv, r, paged_tiles(kv));
            __syncwarp();                                  // every lane is done with the rows before
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                const __half* const row = paged_row(kv, o, q, head, i);
                const uint2 raw = row ? __ldcg(reinterpret_cast<const uint2*>(row) + lane) : make_uint2(0u, 0u);
                sts_v2(xs + i * (kGroup * 2) + lane * 8, raw.x, raw.y);
            }
            __syncwarp();
        }
        float acc[kV][kChains] = {};
        fused_group<kV, true, true>(cur, tb, bits, T, xs, there, acc);
        float* const dst = d_scores + (static_cast<int64_t>(head) * kv.max_tiles + tile) * (kV * 32) + lane;
#pragma unroll
        for (int i = 0; i < kV; ++i) dst[i * 32] = sum_of(acc[i]);
    });
}
template <int kMaxWarps>
__global__ void __launch_bounds__(kMaxWarps * 32, 1)
ecco_paged_scores_mma_kernel(const __grid_constant__ PagedKv kv, const __grid_constant__ PagedOut o, float* __restrict__ d_scores)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    int32_t* const firsts = reinterpret_cast<int32_t*>(smem + 64);
    release_dependents();
    const DecodeTables tb = plan_decode_tables(smem_u32(smem), kv.k_meta, false);    // one symbol per lookup: the tiles need the room
    const int nw = static_cast<int>(decode_warps(tb, kTiledWarpBytes));
    const int lane = static_cast<int>(threadIdx.x & 31u), warp = static_cast<int>(threadIdx.x >> 5);
    const uint32_t tiles_at = tb.warp_base + warp * kTiledWarpBytes;
    issue_decode_tables(tb, kv.k_meta);
    if (!finish_decode_tables(tb)) return;
    dependency_wait();
    fetch_firsts(kv, firsts);
    const float T = tb.T;
    uint32_t vfrag[16];                                    // as load_vfrag has them: row lane / 4
    walk_tiles(kv, firsts, nw, [&](const Block& cur, bool there, int32_t head, int32_t tile, int r, bool other) {
        if (other) {
            const PagedReq q = paged_req(kv, r, paged_tiles(kv));
            const __half* const row = (lane >> 2) < o.score_rows ? paged_row(kv, o, q, head, lane >> 2) : nullptr;
            const uint2* const p = reinterpret_cast<const uint2*>(row) + (lane & 3);
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const uint2 v = row ? __ldcg(p + c * 4) : make_uint2(0u, 0u);
                vfrag[2 * c] = v.x;
                vfrag[2 * c + 1] = v.y;
            }
        }
        float acc[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        row_dot_mma<true, true>(cur, tb, tiles_at, T, there,
                                [&](uint32_t (&v)[16]) {
#pragma unroll
                                    for (int i = 0; i < 16; ++i) v[i] = vfrag[i];
                                }, acc);
        float* const dst = d_scores + (static_cast<int64_t>(head) * kv.max_tiles + tile) * (o.score_rows * 32);
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = 16 * mt + (lane >> 2) + (i >= 2 ? 8 : 0), row = (lane & 3) * 2 + (i & 1);
                if (row < o.score_rows) dst[row * 32 + t] = acc[mt][i];
            }
    });
}

// ---------------------------------------------------------------------------------------------
// K6a: attention of requests of few rows (new tokens x query heads per KV head): single tokens, drafted tokens.
// All tiles of all heads form one line, which is cut into equal runs, one per warp, whatever the requests' lengths: a warp is
// alone from its first tile to its last.  It keeps a ring of tiles in shared memory, filled by bulk copies, and does
//   S = Q K^T (16 rows x 32 tokens a tile, mma.sync), the softmax on the way in fp32, O += P V
// with P taken from the scores' registers as they are.  A piece of a request that lies in one run as a whole is written out; the others
// leave sums and maxima in the workspace and are joined by ecco_paged_join_kernel.
// Bound by memory: 512 bytes per token and KV head (2.1 M tokens and KV heads, 1.09 GB, twelve or sixteen rows: 189 us = 5.75 TB/s, 89 % of the copy
// rate, some of it from L2; scores given, eight rows, 0.61 GB: 111 us = 5.5 TB/s).  The products take nearly as long at sixteen rows, mma.sync being
// slow here, so requests of more rows are for ecco_paged_many_kernel (20 to 32 rows took 57 us here with two tiles of rows, 42 there).
// ---------------------------------------------------------------------------------------------
constexpr int kFewRows = 16;
template <bool kScores> constexpr int kFewWarps = kScores ? 8 : 6;
// Of a stage of a warp's ring, and their number: K and V, or V and scores of up to eight rows.
constexpr int kScoreRows = 8;
template <bool kScores> constexpr uint32_t kFewTileBytes = kScores ? kKvTileBytes + kScoreRows * 128 : 2 * kKvTileBytes;
template <bool kScores> constexpr int kFewStages = kScores ? 3 : 2;
template <bool kScores> constexpr uint32_t kFewWarpBytes = kFewStages<kScores> * kFewTileBytes<kScores> + (kScores ? 0 : kFewRows * 256);
template <bool kScores> constexpr uint32_t kFewSmemBytes = kFewWarps<kScores> * kFewWarpBytes<kScores> + 1024;
// Runs of the line: one per warp, but of three tiles, or joining costs more than waiting (16 requests of 4 to 8 drafted tokens, 2048 tiles: 158
// us with runs of two or three tiles, 145 with three), unless there are so few tiles that every run has just one (2 requests of 780 tokens,
// 400 tiles: 24.4 us with runs of three, 20.4 with runs of one).
constexpr int kFewRunTiles = 3;
template <bool kScores>
__device__ __forceinline__ UnitSplit few_split(int64_t units, int ctas)
{
    const int64_t runs = units <= static_cast<int64_t>(ctas) * 3 ? units : max(units / kFewRunTiles, static_cast<int64_t>(ctas) * 2);
    return UnitSplit(units, static_cast<int>(max(static_cast<int64_t>(1), min(static_cast<int64_t>(ctas) * kFewWarps<kScores>, runs))));
}

// Weights enter the tensor cores as one fp16 number each: half a step, 2^-11 of a weight, is 2^-11 sum p |v| of an output, beside the 2^-11 |out|
// that the output's own rounding costs (measured against 64 bits, norms: 2.2e-4 of the output instead of 2.1e-4 with few rows, 2.8e-4 with
// many).  Two numbers as in ecco_attn_values would leave the latter alone, for half as many products again.  Their sum is taken in fp32 before the
// rounding.  They stand at 2^15 times what they are: taken as they are, those below 6e-5 would lose bits and those below 3e-8 vanish.
constexpr float kWeightLog2 = 15.0f;
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// natural logarithm of a sum of weights that stands at l * 2^(m - offset); NaN where the scores were
__device__ __forceinline__ float lse_of(float m, float l, float offset)
{
    return l == 0.0f ? -INFINITY : (m - offset + log2f(l)) * 0.693147180559945309f;
}
// what a row's sums are multiplied by: zero for a row that has seen nothing
__device__ __forceinline__ float inverse_of(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }
__device__ __forceinline__ uint32_t pack_h2(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// 128 bytes that nobody will read any more before they are written again
__device__ __forceinline__ void discard_line(const uint8_t* p) { asm volatile("discard.global.L2 [%0], 128;" ::"l"(p) : "memory"); }
// bounded wait of a warp on one of its barriers
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity)
{
    bool done = false;
    for (int i = 0; i < 2 * kWaitLimit && !done; ++i) done = mbar_try_wait(bar, parity);
    done = __all_sync(0xffffffffu, done);
    if (!done && (threadIdx.x & 31u) == 0) atomicExch(&g_device_status, ECCO_ERR_DEVICE_TIMEOUT);
    return done;
}

// kScores: the products with K are there already (K6k), only V is in tiles.
template <bool kScores>
__global__ void __launch_bounds__(kFewWarps<kScores> * 32, 1)
ecco_paged_few_kernel(const __grid_constant__ PagedKv kv, const __grid_constant__ PagedOut o, const __grid_constant__ PagedSchedule sc)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    constexpr unsigned full = 0xffffffffu;
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint32_t mine = smem_u32(smem) + 1024 + warp * kFewWarpBytes<kScores>, q_at = mine + kFewStages<kScores> * kFewTileBytes<kScores>;
    const uint32_t bar = smem_u32(smem) + warp * kFewStages<kScores> * 8;
    if (lane == 0)
        for (int s = 0; s < kFewStages<kScores>; ++s) mbar_init(bar + s * 8, 1);
    __syncwarp();
    // Behind ecco_paged_many_kernel the wait comes at the end, where the next kernel needs it: that kernel releases this one only when all its
    // threads have waited, so the tiles, the schedule, q and the batch's arrays are in L2, where every read before the wait goes (__ldcg and bulk
    // copies, no plain loads), and the two kernels write nothing that the other reads or writes.  Waiting here instead, a CTA would begin
    // when the last one of the other kernel has ended and not when its SM is free (24 requests of which six are pieces of prompts: 177 -> 196 us; 8 of
    // 3 to 64 rows over 700 to 1500 tokens: 77 -> 91).
    if (!o.early) dependency_wait();
    release_dependents();
    const int32_t T = paged_tiles(kv), line = __ldcg(sc.few_tiles + kv.n_req);
    // Fewer runs than warps are spread over the CTAs, but behind ecco_paged_many_kernel they go to the first CTAs, which begin earlier.
    const int wg = static_cast<int>(o.early ? blockIdx.x * kFewWarps<kScores> + warp : warp * gridDim.x + blockIdx.x);
    const int64_t U = static_cast<int64_t>(line) * kv.heads;
    const UnitSplit split = few_split<kScores>(U, static_cast<int>(gridDim.x));
    const int64_t u0 = min(split.begin(wg), U), u1 = min(split.begin(wg + 1), U);     // warps beyond the runs: nothing

    // a place in the run: unit u is tile `tile` of head `head`; the request it belongs to has units [begin, end), cut to the run's end
    struct Place { int64_t u, begin, end; int32_t head, tile; PagedReq q; };
    auto seek = [&](Place& p) {
        if (p.u >= u1) return;
        const int32_t nth = static_cast<int32_t>(divide(static_cast<uint64_t>(p.u), static_cast<uint64_t>(line)));
        const int64_t head_from = static_cast<int64_t>(nth) * line;
        p.head = kv.heads - 1 - nth;                       // the last head's tiles are the latest in the L2 cache
        const int r = warp_find(sc.few_tiles, kv.n_req, static_cast<int32_t>(p.u - head_from));
        p.q = paged_req(kv, r, T);
        const int32_t from = __ldcg(sc.few_tiles + r), to = __ldcg(sc.few_tiles + r + 1);
        p.q.tiles = to - from;                             // as many as the line has: the run that has the last of them is one that there is
        p.begin = head_from + from;
        p.end = min(head_from + to, u1);
        p.tile = p.q.first + static_cast<int32_t>(p.u - p.begin);
    };
    Place load = {};                                       // the next tile to ask for
    load.u = u0;
    seek(load);
    Place at = load;                                       // the tile at hand
    uint32_t asked = 0, taken = 0;
    auto ask = [&]() {
        if (load.u >= u1) return;
        if (lane == 0) {
            const uint32_t s = asked % kFewStages<kScores>, b = bar + s * 8, dst = mine + s * kFewTileBytes<kScores>;
            if (kScores) {
                mbar_expect_tx(b, kKvTileBytes + o.score_rows * 128);
                bulk_g2s(dst, staged_tile(kv, 0, load.head, load.tile), kKvTileBytes, b);
                bulk_g2s(dst + kKvTileBytes, o.scores + (static_cast<int64_t>(load.head) * kv.max_tiles + load.tile) * o.score_rows * 32, o.score_rows * 128, b);
            } else {
                mbar_expect_tx(b, 2 * kKvTileBytes);
                bulk_g2s(dst, staged_tile(kv, 0, load.head, load.tile), kKvTileBytes, b);
                bulk_g2s(dst + kKvTileBytes, staged_tile(kv, 1, load.head, load.tile), kKvTileBytes, b);
            }
        }
        ++asked;
        ++load.tile;
        if (++load.u == load.end) seek(load);
    };
    for (int s = 0; s < kFewStages<kScores>; ++s) ask();

    const uint32_t col = (lane & 3u) * 2;
    int32_t cut_rows = 0, cut_place = 0, cut_out = 0, cut_last = 0;    // at most one request begins here and goes on in the next run; lane i: its row i
    bool ok = true;
    while (ok && at.u < u1) {
        const PagedReq q = at.q;
        const int R = min(q.rows * o.q_per_kv, kFewRows);
        const bool whole = at.u == at.begin && at.end - at.u == q.tiles;
        const bool starts = at.u == at.begin;              // the request begins in this run
        const int slot = 2 * wg + (at.u == u0 ? 0 : 1);
        if (starts && !whole) {
            const int row = min(static_cast<int>(lane), R - 1), token = row / o.q_per_kv, hq = (kv.head0 + at.head) * o.q_per_kv + row - token * o.q_per_kv;
            cut_rows = R;
            cut_place = slot * kFewRows + row;
            cut_out = (q.row0 + token) * o.q_heads + hq;
            cut_last = split.owner(at.begin + q.tiles - 1);
        }
        if (!kScores) {
            // the rows of q as tiles: rows beyond the last are zero
            __syncwarp();
            uint4 rows[8];                                 // sixteen lanes to a row, two rows at a time, all on their way together
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int row = 2 * i + static_cast<int>(lane >> 4), token = row / o.q_per_kv, g = row - token * o.q_per_kv;
                rows[i] = make_uint4(0u, 0u, 0u, 0u);
                if (row < R) rows[i] = __ldcg(reinterpret_cast<const uint4*>(o.q + (q.row0 + token) * o.q_stride + (static_cast<int64_t>(kv.head0 + at.head) * o.q_per_kv + g) * kGroup) + (lane & 15u));
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                sts_v4(q_at + ((lane & 15u) >> 1) * 512 + tile_byte(2 * i + (lane >> 4), (lane & 1u) * 8), rows[i].x, rows[i].y, rows[i].z, rows[i].w);
            __syncwarp();
        }
        float acc[16][4], m[2], l[2];
        int32_t seen[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = static_cast<int>(lane >> 2) + 8 * i;
            seen[i] = row < R ? tokens_seen(q, row / o.q_per_kv, o.causal) : 0;
            m[i] = -INFINITY;
            l[i] = 0.0f;
        }
#pragma unroll
        for (int n = 0; n < 16; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[n][i] = 0.0f;

        for (; at.u < at.end; ++at.u, ++at.tile) {
            const uint32_t s = taken % kFewStages<kScores>, k_tile = mine + s * kFewTileBytes<kScores>, v_tile = kScores ? k_tile : k_tile + kKvTileBytes;
            ok = warp_wait(bar + s * 8, (taken / kFewStages<kScores>) & 1u);
            if (!ok) break;
            ++taken;
            // scores: rows x 8 tokens per fragment
            float s4[4][4];
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) s4[n][i] = 0.0f;
            if (kScores) {
                const uint32_t row = lane >> 2;            // the scores of rows that there are not are not looked at
                if (row < static_cast<uint32_t>(o.score_rows))
#pragma unroll
                    for (int n = 0; n < 4; ++n)
                        asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(s4[n][0]), "=f"(s4[n][1]) : "r"(k_tile + kKvTileBytes + row * 128 + (n * 8 + col) * 4));
            } else {
                const uint32_t k_at = k_tile + tile_byte((lane & 7u) + ((lane >> 4) & 1u) * 8, ((lane >> 3) & 1u) * 8);
                const uint32_t a_at = q_at + tile_byte((lane & 7u) + ((lane >> 3) & 1u) * 8, (lane >> 4) * 8);
#pragma unroll
                for (int d = 0; d < 8; ++d) {
                    uint32_t b[2][4];
                    ldmatrix_x4(b[0], k_at + d * kPieceBytes);
                    ldmatrix_x4(b[1], k_at + d * kPieceBytes + 512);
                    uint32_t a[4];
                    ldmatrix_x4(a, a_at + d * 512);
#pragma unroll
                    for (int n = 0; n < 4; ++n) mma_16816(s4[n], a, b[n >> 1][(n & 1) * 2], b[n >> 1][(n & 1) * 2 + 1]);
                }
            }
            // softmax: relative to the largest score so far
            const int32_t t0 = (at.tile - q.first) * 32 + static_cast<int32_t>(col);
            uint32_t p[2][4];                              // A fragments of 16 tokens each
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float top = m[i];
#pragma unroll
                for (int n = 0; n < 4; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float& x = s4[n][2 * i + e];
                        x = t0 + n * 8 + e < seen[i] ? x * o.scale_log2 : -INFINITY;
                        top = fmaxf(top, x);
                    }
                top = fmaxf(top, __shfl_xor_sync(full, top, 1));
                top = fmaxf(top, __shfl_xor_sync(full, top, 2));
                const float base = top == -INFINITY ? 0.0f : top;              // a row that has seen nothing: all weights zero
                if (__any_sync(full, top > m[i])) {
                    const float f = exp2_fast(m[i] - base);
                    l[i] *= f;
#pragma unroll
                    for (int n = 0; n < 16; ++n) { acc[n][2 * i] *= f; acc[n][2 * i + 1] *= f; }
                }
                m[i] = top;
#pragma unroll
                for (int n = 0; n < 4; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float& x = s4[n][2 * i + e];
                        x = exp2_fast(x - base + kWeightLog2);
                        l[i] += x;
                    }
            }
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                p[n >> 1][(n & 1) * 2] = pack_h2(s4[n][0], s4[n][1]);
                p[n >> 1][(n & 1) * 2 + 1] = pack_h2(s4[n][2], s4[n][3]);
            }
            const uint32_t v_at = v_tile + tile_byte((lane & 7u) + ((lane >> 3) & 1u) * 8, (lane >> 4) * 8);
#pragma unroll
            for (int d = 0; d < 8; ++d)
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    uint32_t b[4];
                    ldmatrix_x4_trans(b, v_at + d * kPieceBytes + ks * 512);
                    mma_16816(acc[2 * d], p[ks], b[0], b[1]);
                    mma_16816(acc[2 * d + 1], p[ks], b[2], b[3]);
                }
            __syncwarp();                                  // the whole warp has read the tile
            if (o.discard) {
                // nobody reads the tile again: what of it is still in the L2 cache need not go to memory (1.06 M tokens and KV heads:
                // 273 -> 260 us, 2.1 M: 533 -> 522)
#pragma unroll
                for (int i = 0; i < (kScores ? 2 : 4); ++i) discard_line(staged_tile(kv, i >> 1, at.head, at.tile) + (i & 1) * (kKvTileBytes / 2) + lane * 128);
            }
            ask();
        }
        // out, or into a slot
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float sum = l[i];
            sum += __shfl_xor_sync(full, sum, 1);
            sum += __shfl_xor_sync(full, sum, 2);
            const int row = static_cast<int>(lane >> 2) + 8 * i;
            if (row >= R || !ok) continue;
            if (whole) {
                const int token = row / o.q_per_kv, hq = (kv.head0 + at.head) * o.q_per_kv + row - token * o.q_per_kv;
                const int64_t at_row = static_cast<int64_t>(q.row0 + token) * o.q_heads + hq;
                const float inv = inverse_of(sum);
                uint32_t* const dst = reinterpret_cast<uint32_t*>(o.out + at_row * kGroup) + (lane & 3u);
#pragma unroll
                for (int n = 0; n < 16; ++n) dst[n * 4] = pack_h2(acc[n][2 * i] * inv, acc[n][2 * i + 1] * inv);
                if (o.lse && (lane & 3u) == 0) o.lse[at_row] = lse_of(m[i], sum, kWeightLog2);
            } else {
                const int64_t at_row = static_cast<int64_t>(slot) * kFewRows + row;
                float2* const dst = reinterpret_cast<float2*>(o.part + at_row * kGroup) + (lane & 3u);
#pragma unroll
                for (int n = 0; n < 16; ++n) dst[n * 4] = make_float2(acc[n][2 * i], acc[n][2 * i + 1]);
                if ((lane & 3u) == 0) o.part_ml[at_row] = make_float2(m[i], sum);
            }
        }
        if (ok) seek(at);
    }
    if (ok && cut_rows) {
        int32_t n = 0;
        if (lane == 0) n = atomicAdd(o.n_cuts, cut_rows);
        n = __shfl_sync(full, n, 0);
        if (static_cast<int32_t>(lane) < cut_rows) o.cuts[n + lane] = FewCut{cut_out, cut_place, wg, cut_last};
    }
    if (o.early) dependency_wait();
    if (!ok)                                               // tiles on their way land before the warp leaves
        for (; taken < asked; ++taken) warp_wait(bar + (taken % kFewStages<kScores>) * 8, (taken / kFewStages<kScores>) & 1u);
}

// adds a piece's sums v, with maximum and sum of weights x, to those at hand; a piece that has seen nothing has sums of zero
__device__ __forceinline__ void join_sums(float& m, float& l, float4& acc, float2 x, float4 v)
{
    const float top = fmaxf(m, x.y == 0.0f ? -INFINITY : x.x), base = top == -INFINITY ? 0.0f : top;
    const float f0 = exp2_fast(m - base), f1 = x.y == 0.0f ? 0.0f : exp2_fast(x.x - base);
    l = l * f0 + x.y * f1;
    acc = make_float4(acc.x * f0 + v.x * f1, acc.y * f0 + v.y * f1, acc.z * f0 + v.z * f1, acc.w * f0 + v.w * f1);
    m = top;
}
// Joins the pieces of the rows of cut requests.  A row has as many warps as there are for it, up to eight, and these share the pieces.  The order
// of the rows is that in which ecco_paged_few_kernel came to them, but what happens to a row depends on their number alone.
// Waits for memory, so the rows are spread over all warps that find room at once (with a CTA to each run, most of which had nothing to join,
// 16 requests of 4 to 8 drafted tokens took 147 us instead of 142, 8 of 3 to 64 over 700 to 1500 tokens 90 instead of 85).
constexpr int kJoinCtas = 3;                               // per SM: as many as fit
__global__ void __launch_bounds__(256, kJoinCtas)
ecco_paged_join_kernel(const __grid_constant__ PagedOut o)
{
    __shared__ float4 sums[8][32];
    __shared__ float2 ml[8];
    const int lane = static_cast<int>(threadIdx.x & 31u), warp = static_cast<int>(threadIdx.x >> 5);
    release_dependents();
    dependency_wait();
    const int32_t n = __ldcg(o.n_cuts), warps = static_cast<int32_t>(gridDim.x) * 8;
    const int team = n <= warps / 8 ? 8 : n <= warps / 4 ? 4 : n <= warps / 2 ? 2 : 1, sub = warp % team;
    for (int32_t first = static_cast<int32_t>(blockIdx.x) * (8 / team); first < n; first += warps / team) {
        const bool there = first + warp / team < n;
        const int4 c = there ? __ldcg(reinterpret_cast<const int4*>(o.cuts + first + warp / team)) : make_int4(0, 0, 0, -1);
        const int row = c.y % kFewRows, w_lo = c.z, w_hi = c.w;
        float m = -INFINITY, l = 0.0f;
        float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 1
        for (int w0 = w_lo + sub; w0 <= w_hi; w0 += 8 * team) {                      // eight pieces on their way together
            float2 x[8];
            float4 v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int w = min(w0 + k * team, w_hi);
                const int64_t at = w == w_lo ? c.y : static_cast<int64_t>(2 * w) * kFewRows + row;
                x[k] = __ldcg(o.part_ml + at);
                v[k] = __ldcg(reinterpret_cast<const float4*>(o.part + at * kGroup) + lane);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (w0 + k * team <= w_hi) join_sums(m, l, acc, x[k], v[k]);
        }
        if (team > 1) {
            sums[warp][lane] = acc;
            if (lane == 0) ml[warp] = make_float2(m, l);
            __syncthreads();
            if (sub == 0)
                for (int w = warp + 1; w < warp + team; ++w) join_sums(m, l, acc, ml[w], sums[w][lane]);
            __syncthreads();
        }
        if (sub == 0 && there) {
            const float inv = inverse_of(l);
            reinterpret_cast<uint2*>(o.out + static_cast<int64_t>(c.x) * kGroup)[lane] = make_uint2(pack_h2(acc.x * inv, acc.y * inv), pack_h2(acc.z * inv, acc.w * inv));
            if (o.lse && lane == 0) o.lse[c.x] = lse_of(m, l, kWeightLog2);
        }
    }
}

}  // namespace
