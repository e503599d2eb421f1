// ecco_kernels.cu -- sm_100a kernels and the device half of the C ABI.
//
// One thread owns one group: a 64-byte block is independent of every other block (Sec. 3.2,
// "all group-wise information ... compressed to a fixed compressed block size"), so the decoder
// runs the serial Huffman chain (Sec. 4.2) once per thread and takes its parallelism across
// groups, not inside a group.  The lanes of a warp advance symbol by symbol in lock step, which
// keeps every per-symbol index (output position, activation element) uniform across the warp.
//
// Shared memory per CTA (sizes from the image's header, see ecco_decode_core.cuh):
//   tables   pattern[64][16] fp16 | codebook records [256] x 16 B | pair tables | centroids in rank order [256][16] fp16 | shape tables
//            [n_shapes][256] u8, and behind the warps' arrays, at the end of shared memory, ID_KP table [4096] u16; all but the centroids
//            are brought in by bulk copies (cp.async.bulk + mbarrier)
//   per warp bits[19][32] u32   the warp's 32 blocks, word-transposed: lane L's word w at
//                               [w][L] -> bank L whatever w is (conflict-free refills);
//                               rows 16 to 18 are scratch: what a lane reads past stream bit 512 does not matter (decode_group).  The
//                               scalar fused kernels keep the decoded ranks over its consumed rows, for the outlier fix-up
//            tiles              ecco_decompress: one [32 groups][16 values] fp16 staging tile for the tensor stores;
//                               tensor-core kernels: eight of them, the whole decoded group, as MMA operands
//
// Layout of the sources (one translation unit; the .cuh files are included here and nowhere else):
//   ecco_device_core.cuh            PTX helpers, bounded waits, overlapped launches
//   ecco_decode_core.cuh            the group decoder with the value table in registers
//   ecco_decompress_kernels.cuh     ecco_decompress (tile-store and small-tensor kernels), ecco_var_decompress
//   ecco_fused_scalar_kernels.cuh   fused GEMV (one to five rows) / attention scores (one or two heads)
//   ecco_group_tiles.cuh            decoded groups as fp16 tiles in shared memory
//   ecco_fused_mma_kernels.cuh      the same for more rows and heads, on the tensor cores
//   ecco_attn_values_kernels.cuh    softmax(scores) . V over a compressed V cache
//   ecco_act2x_kernels.cuh          2x activation codec
//   ecco_kv_compress_kernel.cuh     online 4x compressor
//   ecco_paged_kernels.cuh          paged KV cache: slots and block tables, pages into tiles, attention of few rows
//   ecco_paged_many_kernel.cuh      attention of many rows over it, on tcgen05
//   ecco_rope_kernels.cuh           rotary positions
//   ecco_paged8_core.cuh            the format of a paged KV cache in 8 bits
//   ecco_paged8_kernels.cuh         append to it, attention of few rows over it
//   ecco_launch.cuh                 device query, overlapped launches, work plans
//   this file                       the C ABI: argument checks and launches
#include "ecco_device_core.cuh"
#include "ecco_decode_core.cuh"
#include "ecco_decompress_kernels.cuh"
#include "ecco_fused_scalar_kernels.cuh"
#include "ecco_group_tiles.cuh"
#include "ecco_attn_values_kernels.cuh"
#include "ecco_fused_mma_kernels.cuh"
#include "ecco_launch.cuh"
#include "ecco_act2x_kernels.cuh"
#include "ecco_kv_compress_kernel.cuh"
#include "ecco_paged_kernels.cuh"
#include "ecco_paged8_core.cuh"
#include "ecco_paged_many_kernel.cuh"
#include "ecco_rope_kernels.cuh"
#include "ecco_paged8_kernels.cuh"


// ---------------------------------------------------------------------------------------------
// C ABI
// ---------------------------------------------------------------------------------------------
extern "C" int ecco_last_cuda_error(void) { return t_last_cuda_error; }
extern "C" uint64_t ecco_kernel_launch_count(void) { return g_launches.load(); }

extern "C" int ecco_device_status(void)
{
    cudaError_t e = cudaDeviceSynchronize();
    if (e != cudaSuccess) { t_last_cuda_error = static_cast<int>(e); return ECCO_ERR_CUDA; }
    int st = 0, zero = 0;
    e = cudaMemcpyFromSymbol(&st, g_device_status, sizeof st);
    if (e == cudaSuccess && st) e = cudaMemcpyToSymbol(g_device_status, &zero, sizeof zero);
    if (e != cudaSuccess) { t_last_cuda_error = static_cast<int>(e); return ECCO_ERR_CUDA; }
    return st;
}

// Diagnostics: the give-up path of the bounded wait, exercised without anything that could hang.  The kernel arms a
// barrier with a byte count that no copy will ever deliver (nothing is in flight, so the CTA may exit at any time),
// polls it a few hundred times, gives up, records the time-out and returns normally.
namespace {
__global__ void ecco_wait_timeout_probe_kernel()
{
    __shared__ __align__(8) uint64_t bar;
    const uint32_t b = smem_u32(&bar);
    if (threadIdx.x == 0) {
        mbar_init(b, 1);
        mbar_expect_tx(b, 64);
    }
    (void)bounded_wait(b, 0, 256);
}
}  // namespace
extern "C" int ecco_test_wait_timeout(void* stream)
{
    DeviceInfo di;
    int rc = device_info(&di);
    if (rc) return rc;
    ecco_wait_timeout_probe_kernel<<<1, 64, 0, static_cast<cudaStream_t>(stream)>>>();
    return check_launch();
}

// cuTensorMapEncodeTiled through the runtime's driver entry point query (no link against libcuda)
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeTiledFn encode_tiled_fn()
{
    static std::once_flag once;
    static EncodeTiledFn fn = nullptr;
    std::call_once(once, [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(p);
    });
    return fn;
}

// tensor map of the output seen as [n_groups][128] fp16, box = 32 rows x 16 values, 32-byte swizzle
static bool make_out_map(CUtensorMap* map, void* d_out, uint64_t n_groups)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {kGroup, n_groups};
    const cuuint64_t strides[1] = {kGroup * 2};
    const cuuint32_t box[2] = {16, 32};
    const cuuint32_t estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, d_out, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_32B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr int kDecompressTmaWarps = 32;

// every decoding kernel asks for all the shared memory of an SM and lays itself out on the device
template <class K>
static int want_all_smem(K kernel, bool* configured)
{
    if (*configured) return ECCO_OK;
    const int rc = set_smem(kernel, kSmemCtaBytes);
    if (rc == ECCO_OK) *configured = true;
    return rc;
}

// tensors of fewer than 32 groups (the tile store's box is 32 rows tall), or when no tensor map can be made
static int launch_decompress_small(const DeviceInfo& di, const void* d_meta, const uint8_t* d_blocks, uint64_t n_groups, void* d_out,
                                   cudaStream_t stream)
{
    static thread_local bool configured[64] = {};
    auto kernel = ecco_decompress_kernel<kDecompressWarps>;
    int rc = want_all_smem(kernel, &configured[di.device]);
    if (rc) return rc;
    const unsigned grid = static_cast<unsigned>(spread_ctas(static_cast<int64_t>((n_groups + 31) / 32), di.sms));
    kernel<<<grid, kDecompressWarps * 32, kSmemCtaBytes, stream>>>(static_cast<const uint8_t*>(d_meta), d_blocks, n_groups,
                                                                   static_cast<uint16_t*>(d_out));
    return check_launch();
}

// one launch of the tile-store kernel over batch.n tensors (maps already made)
static int launch_decompress_batch(const DeviceInfo& di, DecompressBatch& batch, cudaStream_t stream)
{
    static thread_local bool configured[64] = {};
    auto kernel = ecco_decompress_tma_kernel<kDecompressTmaWarps>;
    int rc = want_all_smem(kernel, &configured[di.device]);
    if (rc) return rc;
    uint64_t tiles = 0;
    for (int t = 0; t < batch.n; ++t) tiles += (batch.job[t].n_groups + 31) / 32;
    const unsigned grid = static_cast<unsigned>(spread_ctas(static_cast<int64_t>(tiles), di.sms));
    return launch_overlapped(kernel, grid, spread_threads(static_cast<int64_t>(tiles), static_cast<int>(grid), kDecompressTmaWarps), kSmemCtaBytes, stream, batch);
}

// The tile-store kernel addresses output rows with the 32-bit signed coordinates of the TMA unit: tensors of 2^31 groups
// (256 GiB of fp16) or more are refused.
constexpr uint64_t kMaxGroups = (1ull << 31) - 32;

static int check_decompress_args(const void* d_meta, const uint8_t* d_blocks, uint64_t n_groups, const void* d_out)
{
    if (!d_meta || !d_blocks || !d_out) return ECCO_ERR_INVALID_ARG;
    if (!aligned16(d_meta) || !aligned16(d_blocks) || !aligned16(d_out)) return ECCO_ERR_ALIGNMENT;
    if (n_groups > kMaxGroups) return ECCO_ERR_INVALID_ARG;
    return ECCO_OK;
}

extern "C" int ecco_decompress_batch(const ecco_decompress_item* items, int32_t n_items, void* stream)
{
    if (n_items < 0 || (n_items > 0 && !items)) return ECCO_ERR_INVALID_ARG;
    for (int i = 0; i < n_items; ++i) {                    // nothing is launched unless every item is acceptable
        if (items[i].n_groups == 0) continue;
        const int rc = check_decompress_args(items[i].d_meta, items[i].d_blocks, items[i].n_groups, items[i].d_out_fp16);
        if (rc) return rc;
    }
    DeviceInfo di;
    int rc = device_info(&di);
    if (rc) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    DecompressBatch batch;
    std::memset(&batch, 0, sizeof batch);
    for (int i = 0; i < n_items; ++i) {
        const ecco_decompress_item& it = items[i];
        if (it.n_groups == 0) continue;
        DecompressJob& job = batch.job[batch.n];
        if (it.n_groups >= 32 && make_out_map(&job.map, it.d_out_fp16, it.n_groups)) {
            job.meta = static_cast<const uint8_t*>(it.d_meta);
            job.blocks = it.d_blocks;
            job.n_groups = it.n_groups;
            job.out = static_cast<uint16_t*>(it.d_out_fp16);
            if (++batch.n == kMaxJobs) {
                rc = launch_decompress_batch(di, batch, s);
                if (rc) return rc;
                batch.n = 0;
            }
        } else {                                           // items keep their order in the stream
            if (batch.n) {
                rc = launch_decompress_batch(di, batch, s);
                if (rc) return rc;
                batch.n = 0;
            }
            rc = launch_decompress_small(di, it.d_meta, it.d_blocks, it.n_groups, it.d_out_fp16, s);
            if (rc) return rc;
        }
    }
    return batch.n ? launch_decompress_batch(di, batch, s) : ECCO_OK;
}

extern "C" int ecco_decompress(const void* d_meta, const uint8_t* d_blocks, uint64_t n_groups, void* d_out, void* stream)
{
    if (n_groups == 0) return ECCO_OK;
    const ecco_decompress_item item = {d_meta, d_blocks, n_groups, d_out};
    return ecco_decompress_batch(&item, 1, stream);
}

constexpr int kVarWarps = 28;

extern "C" int ecco_var_decompress(const void* d_meta, const uint8_t* d_stream, const void* d_index, uint64_t n_groups, void* d_out,
                                   void* stream)
{
    if (n_groups == 0) return ECCO_OK;
    if (!d_meta || !d_stream || !d_index || !d_out) return ECCO_ERR_INVALID_ARG;
    if (!aligned16(d_meta) || !aligned16(d_stream) || !aligned16(d_out) || (reinterpret_cast<uintptr_t>(d_index) & 7u)) return ECCO_ERR_ALIGNMENT;
    if (n_groups > kMaxGroups) return ECCO_ERR_INVALID_ARG;
    DeviceInfo di;
    int rc = device_info(&di);
    if (rc) return rc;
    // rows past the end of the tensor are dropped by the tile store, so any n_groups >= 1 works
    CUtensorMap map;
    if (!make_out_map(&map, d_out, n_groups)) return ECCO_ERR_CUDA;
    auto kernel = ecco_var_decompress_kernel<kVarWarps>;
    static thread_local bool configured[64] = {};
    rc = want_all_smem(kernel, &configured[di.device]);
    if (rc) return rc;
    const unsigned grid = static_cast<unsigned>(spread_ctas(static_cast<int64_t>((n_groups + 31) / 32), di.sms));
    return launch_overlapped(kernel, grid, spread_threads(static_cast<int64_t>((n_groups + 31) / 32), static_cast<int>(grid), kVarWarps), kSmemCtaBytes, static_cast<cudaStream_t>(stream),
                             static_cast<const uint8_t*>(d_meta), reinterpret_cast<const uint4*>(d_stream),
                             static_cast<const uint64_t*>(d_index), n_groups, map);
}

extern "C" size_t ecco_gemv_workspace_bytes(int32_t n_out, int32_t k, int32_t batch)
{
    if (n_out <= 0 || k <= 0 || k % kGroup || batch < 1 || batch > ECCO_MAX_BATCH) return 0;
    // sized for the largest plan any supported device can ask for (at most 256 persistent CTAs)
    const int row_tiles = (n_out + 31) / 32;
    const GemvPlan p = gemv_plan_for(static_cast<int64_t>(row_tiles) * (k / kGroup), row_tiles, pad_v(batch), 256);
    return p.partial_bytes + p.ticket_bytes;
}

// the matrices of one call with their places in the call's unit and tile spaces
struct GemvCall {
    GemvBatch b;
    int row_tiles;
};
static void gemv_call_begin(GemvCall* c)
{
    std::memset(c, 0, sizeof *c);
}
static void gemv_call_add(GemvCall* c, const void* d_meta, const uint8_t* d_blocks, int n_out, int kblocks, const void* d_x, float* d_y)
{
    GemvJob& j = c->b.job[c->b.n++];
    j.meta = static_cast<const uint8_t*>(d_meta);
    j.blocks = d_blocks;
    j.x = static_cast<const __half*>(d_x);
    j.y = d_y;
    j.n_out = n_out;
    j.kblocks = kblocks;
    j.tile_first = c->row_tiles;
    j.unit_first = c->b.units;
    const int tiles = (n_out + 31) / 32;
    c->row_tiles += tiles;
    c->b.units += static_cast<int64_t>(tiles) * kblocks;
}

// six to eight rows of x: the tensor-core kernel
template <bool kGiveUp = false>
static int launch_gemv_mma_call(const DeviceInfo& di, const GemvCall& c, int batch, void* d_ws, size_t ws_bytes, cudaStream_t stream)
{
    auto kernel = ecco_gemv_mma_kernel<kMmaWarps, kGiveUp>;
    static thread_local bool configured[64] = {};
    int rc = want_all_smem(kernel, &configured[di.device]);
    if (rc) return rc;
    const GemvPlan p = gemv_plan_for(c.b.units, c.row_tiles, 8, di.sms < 256 ? di.sms : 256);
    if (!d_ws || !aligned16(d_ws)) return d_ws ? ECCO_ERR_ALIGNMENT : ECCO_ERR_WORKSPACE;
    if (ws_bytes < p.partial_bytes + p.ticket_bytes) return ECCO_ERR_WORKSPACE;
    float* partial = static_cast<float*>(d_ws);
    Ticket* tickets = reinterpret_cast<Ticket*>(static_cast<uint8_t*>(d_ws) + p.partial_bytes);
    return launch_overlapped(kernel, static_cast<unsigned>(p.grid), spread_threads(c.b.units, p.grid, kMmaWarps), kSmemCtaBytes, stream, c.b, batch,
                             partial, tickets, next_ticket_tag());
}
static int launch_gemv_mma(const DeviceInfo& di, const void* d_meta, const uint8_t* d_blocks, int n_out, int kblocks,
                           const void* d_x, int batch, float* d_y, void* d_ws, size_t ws_bytes, cudaStream_t stream)
{
    GemvCall c;
    gemv_call_begin(&c);
    gemv_call_add(&c, d_meta, d_blocks, n_out, kblocks, d_x, d_y);
    return launch_gemv_mma_call(di, c, batch, d_ws, ws_bytes, stream);
}

// one to five rows of x (batch == kV): the per-warp kernel
template <int kV, bool kGiveUp = false>
static int launch_gemv_warp_call(const DeviceInfo& di, const GemvCall& c, void* d_ws, size_t ws_bytes, cudaStream_t stream)
{
    constexpr int kFusedWarps = gemv_warp_warps(kV);
    auto kernel = ecco_gemv_warp_kernel<kV, kFusedWarps, kGiveUp>;
    static thread_local bool configured[64] = {};
    int rc = want_all_smem(kernel, &configured[di.device]);
    if (rc) return rc;
    const GemvPlan p = gemv_plan_for(c.b.units, c.row_tiles, kV, di.sms < 256 ? di.sms : 256);
    if (!d_ws || !aligned16(d_ws)) return d_ws ? ECCO_ERR_ALIGNMENT : ECCO_ERR_WORKSPACE;
    if (ws_bytes < p.partial_bytes + p.ticket_bytes) return ECCO_ERR_WORKSPACE;
    float* partial = static_cast<float*>(d_ws);
    Ticket* tickets = reinterpret_cast<Ticket*>(static_cast<uint8_t*>(d_ws) + p.partial_bytes);
    return launch_overlapped(kernel, static_cast<unsigned>(p.grid), spread_threads(c.b.units, p.grid, kFusedWarps), kSmemCtaBytes, stream, c.b,
                             partial, tickets, next_ticket_tag());
}
template <int kV>
static int launch_gemv_warp(const DeviceInfo& di, const void* d_meta, const uint8_t* d_blocks, int n_out, int kblocks,
                            const void* d_x, float* d_y, void* d_ws, size_t ws_bytes, cudaStream_t stream)
{
    GemvCall c;
    gemv_call_begin(&c);
    gemv_call_add(&c, d_meta, d_blocks, n_out, kblocks, d_x, d_y);
    return launch_gemv_warp_call<kV>(di, c, d_ws, ws_bytes, stream);
}

extern "C" int ecco_gemv(const void* d_meta, const uint8_t* d_blocks, int32_t n_out, int32_t k, const void* d_x,
                         int32_t batch, float* d_y, void* d_workspace, size_t workspace_bytes, void* stream)
{
    if (!d_meta || !d_blocks || !d_x || !d_y) return ECCO_ERR_INVALID_ARG;
    if (n_out <= 0 || k <= 0 || k % kGroup || batch < 1 || batch > ECCO_MAX_BATCH) return ECCO_ERR_INVALID_ARG;
    if (!aligned16(d_meta) || !aligned16(d_blocks) || !aligned16(d_x) || !aligned16(d_y)) return ECCO_ERR_ALIGNMENT;
    DeviceInfo di;
    int rc = device_info(&di);
    if (rc) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int kblocks = k / kGroup;
    switch (pad_v(batch)) {
        case 1: return launch_gemv_warp<1>(di, d_meta, d_blocks, n_out, kblocks, d_x, d_y, d_workspace, workspace_bytes, s);
        case 2: return launch_gemv_warp<2>(di, d_meta, d_blocks, n_out, kblocks, d_x, d_y, d_workspace, workspace_bytes, s);
        case 3: return launch_gemv_warp<3>(di, d_meta, d_blocks, n_out, kblocks, d_x, d_y, d_workspace, workspace_bytes, s);
        case 4: return launch_gemv_warp<4>(di, d_meta, d_blocks, n_out, kblocks, d_x, d_y, d_workspace, workspace_bytes, s);
        case 5: return launch_gemv_warp<5>(di, d_meta, d_blocks, n_out, kblocks, d_x, d_y, d_workspace, workspace_bytes, s);
        default: return launch_gemv_mma(di, d_meta, d_blocks, n_out, kblocks, d_x, batch, d_y, d_workspace, workspace_bytes, s);
    }
}

// several matrices in one call: one unit space, one launch
static int check_gemv_items(const ecco_gemv_item* items, int32_t n_items, int32_t batch)
{
    if (!items || n_items < 1 || n_items > ECCO_MAX_GEMV_ITEMS || batch < 1 || batch > ECCO_MAX_BATCH) return ECCO_ERR_INVALID_ARG;
    for (int i = 0; i < n_items; ++i) {
        const ecco_gemv_item& it = items[i];
        if (!it.d_meta || !it.d_blocks || !it.d_x_fp16 || !it.d_y) return ECCO_ERR_INVALID_ARG;
        if (it.n_out <= 0 || it.k <= 0 || it.k % kGroup) return ECCO_ERR_INVALID_ARG;
        if (!aligned16(it.d_meta) || !aligned16(it.d_blocks) || !aligned16(it.d_x_fp16) || !aligned16(it.d_y)) return ECCO_ERR_ALIGNMENT;
    }
    return ECCO_OK;
}
static void gemv_call_from_items(GemvCall* c, const ecco_gemv_item* items, int32_t n_items)
{
    gemv_call_begin(c);
    for (int i = 0; i < n_items; ++i)
        gemv_call_add(c, items[i].d_meta, items[i].d_blocks, items[i].n_out, items[i].k / kGroup, items[i].d_x_fp16, items[i].d_y);
}

extern "C" size_t ecco_gemv_batch_workspace_bytes(const ecco_gemv_item* items, int32_t n_items, int32_t batch)
{
    if (!items || n_items < 1 || n_items > ECCO_MAX_GEMV_ITEMS || batch < 1 || batch > ECCO_MAX_BATCH) return 0;
    int64_t units = 0, tiles = 0;
    for (int i = 0; i < n_items; ++i) {
        if (items[i].n_out <= 0 || items[i].k <= 0 || items[i].k % kGroup) return 0;
        const int64_t t = (items[i].n_out + 31) / 32;
        tiles += t;
        units += t * (items[i].k / kGroup);
    }
    if (tiles > INT32_MAX) return 0;
    const GemvPlan p = gemv_plan_for(units, static_cast<int>(tiles), pad_v(batch), 256);
    return p.partial_bytes + p.ticket_bytes;
}

extern "C" int ecco_gemv_batch(const ecco_gemv_item* items, int32_t n_items, int32_t batch, void* d_workspace,
                               size_t workspace_bytes, void* stream)
{
    int rc = check_gemv_items(items, n_items, batch);
    if (rc) return rc;
    DeviceInfo di;
    rc = device_info(&di);
    if (rc) return rc;
    GemvCall c;
    gemv_call_from_items(&c, items, n_items);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    switch (pad_v(batch)) {
        case 1: return launch_gemv_warp_call<1>(di, c, d_workspace, workspace_bytes, s);
        case 2: return launch_gemv_warp_call<2>(di, c, d_workspace, workspace_bytes, s);
        case 3: return launch_gemv_warp_call<3>(di, c, d_workspace, workspace_bytes, s);
        case 4: return launch_gemv_warp_call<4>(di, c, d_workspace, workspace_bytes, s);
        case 5: return launch_gemv_warp_call<5>(di, c, d_workspace, workspace_bytes, s);
        default: return launch_gemv_mma_call(di, c, batch, d_workspace, workspace_bytes, s);
    }
}

extern "C" int ecco_test_gemv_give_up(const ecco_gemv_item* items, int32_t n_items, int32_t batch, void* d_workspace,
                                      size_t workspace_bytes, void* stream)
{
    int rc = check_gemv_items(items, n_items, batch);
    if (rc) return rc;
    if (batch > 1 && pad_v(batch) < 8) return ECCO_ERR_INVALID_ARG;
    DeviceInfo di;
    rc = device_info(&di);
    if (rc) return rc;
    GemvCall c;
    gemv_call_from_items(&c, items, n_items);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return batch == 1 ? launch_gemv_warp_call<1, true>(di, c, d_workspace, workspace_bytes, s)
                      : launch_gemv_mma_call<true>(di, c, batch, d_workspace, workspace_bytes, s);
}

// ---------------------------------------------------------------------------------------------
// ecco_gemv_static_ws: ecco_gemv for callers that cannot allocate.  The split-k scratch is this
// fixed array in the library's device image.  In host code the name below is only a handle for
// the runtime, not a device address: the address comes from cudaGetSymbolAddress, once per
// device, and that pointer is what the kernel receives.
// ---------------------------------------------------------------------------------------------
static __device__ __align__(256) unsigned char g_static_workspace[ECCO_STATIC_WORKSPACE_BYTES];

extern "C" int ecco_gemv_static_ws(const void* d_meta, const uint8_t* d_blocks, int32_t n_out, int32_t k, const void* d_x,
                                   int32_t batch, float* d_y, void* stream)
{
    if (!d_meta || !d_blocks || !d_x || !d_y) return ECCO_ERR_INVALID_ARG;
    if (n_out <= 0 || k <= 0 || k % kGroup || batch < 1 || batch > ECCO_MAX_BATCH) return ECCO_ERR_INVALID_ARG;
    if (!aligned16(d_meta) || !aligned16(d_blocks) || !aligned16(d_x) || !aligned16(d_y)) return ECCO_ERR_ALIGNMENT;
    DeviceInfo di;
    int rc = device_info(&di);
    if (rc) return rc;
    const int kblocks = k / kGroup, vpad = pad_v(batch);
    // refuse, before any launch, a shape whose plan does not fit the fixed array
    const int ctas = di.sms < 256 ? di.sms : 256;
    const int row_tiles = (n_out + 31) / 32;
    const GemvPlan p = gemv_plan_for(static_cast<int64_t>(row_tiles) * kblocks, row_tiles, vpad, ctas);
    if (p.partial_bytes + p.ticket_bytes > ECCO_STATIC_WORKSPACE_BYTES) return ECCO_ERR_WORKSPACE;
    // one-time set-up per device (the current device is di.device): resolve the array's address
    static std::mutex mu;
    static void* address[64] = {};
    void* ws = nullptr;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!address[di.device]) {
            void* ptr = nullptr;
            cudaError_t e = cudaGetSymbolAddress(&ptr, g_static_workspace);
            if (e != cudaSuccess || !ptr) { t_last_cuda_error = static_cast<int>(e); return ECCO_ERR_CUDA; }
            address[di.device] = ptr;
        }
        ws = address[di.device];
    }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    switch (vpad) {
        case 1: return launch_gemv_warp<1>(di, d_meta, d_blocks, n_out, kblocks, d_x, d_y, ws, ECCO_STATIC_WORKSPACE_BYTES, s);
        case 2: return launch_gemv_warp<2>(di, d_meta, d_blocks, n_out, kblocks, d_x, d_y, ws, ECCO_STATIC_WORKSPACE_BYTES, s);
        case 3: return launch_gemv_warp<3>(di, d_meta, d_blocks, n_out, kblocks, d_x, d_y, ws, ECCO_STATIC_WORKSPACE_BYTES, s);
        case 4: return launch_gemv_warp<4>(di, d_meta, d_blocks, n_out, kblocks, d_x, d_y, ws, ECCO_STATIC_WORKSPACE_BYTES, s);
        case 5: return launch_gemv_warp<5>(di, d_meta, d_blocks, n_out, kblocks, d_x, d_y, ws, ECCO_STATIC_WORKSPACE_BYTES, s);
        default: return launch_gemv_mma(di, d_meta, d_blocks, n_out, kblocks, d_x, batch, d_y, ws, ECCO_STATIC_WORKSPACE_BYTES, s);
    }
}

template <int kV>
static int launch_attn(const DeviceInfo& di, const void* d_meta, const uint8_t* d_kblocks, int batch, int n_kv_heads,
                       int seq, const void* d_q, float scale, float* d_scores, cudaStream_t stream)
{
    constexpr int kFusedWarps = fused_warps(kV);
    auto kernel = ecco_attn_scores_kernel<kV, kFusedWarps>;
    static thread_local bool configured[64] = {};
    int rc = want_all_smem(kernel, &configured[di.device]);
    if (rc) return rc;
    const int heads = batch * n_kv_heads;
    // persistent CTAs; the units (32 tokens of a head) are split evenly over the working warps on the device
    const int64_t units = static_cast<int64_t>(heads) * ((seq + 31) / 32);
    const unsigned grid = static_cast<unsigned>(spread_ctas(units, di.sms));
    return launch_overlapped(kernel, grid, spread_threads(units, static_cast<int>(grid), kFusedWarps), kSmemCtaBytes, stream, static_cast<const uint8_t*>(d_meta),
                             d_kblocks, heads, seq, static_cast<const __half*>(d_q), scale, d_scores);
}

extern "C" int ecco_attn_scores(const void* d_meta, const uint8_t* d_kblocks, int32_t batch, int32_t n_kv_heads, int32_t seq,
                                int32_t q_per_kv, const void* d_q, float scale, float* d_scores, void* stream)
{
    if (batch == 0 || n_kv_heads == 0 || seq == 0) return (batch < 0 || n_kv_heads < 0 || seq < 0) ? ECCO_ERR_INVALID_ARG : ECCO_OK;
    if (!d_meta || !d_kblocks || !d_q || !d_scores) return ECCO_ERR_INVALID_ARG;
    if (batch < 0 || n_kv_heads < 0 || seq < 0 || q_per_kv < 1 || q_per_kv > 8) return ECCO_ERR_INVALID_ARG;
    if (static_cast<int64_t>(batch) * n_kv_heads > (1 << 24)) return ECCO_ERR_INVALID_ARG;
    if (!aligned16(d_meta) || !aligned16(d_kblocks) || !aligned16(d_q) || !aligned16(d_scores)) return ECCO_ERR_ALIGNMENT;
    DeviceInfo di;
    int rc = device_info(&di);
    if (rc) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    switch (pad_v(q_per_kv)) {
        case 1: return launch_attn<1>(di, d_meta, d_kblocks, batch, n_kv_heads, seq, d_q, scale, d_scores, s);
        case 2: return launch_attn<2>(di, d_meta, d_kblocks, batch, n_kv_heads, seq, d_q, scale, d_scores, s);
        default: {
            auto kernel = ecco_attn_scores_mma_kernel<kMmaWarps>;
            static thread_local bool configured[64] = {};
            rc = want_all_smem(kernel, &configured[di.device]);
            if (rc) return rc;
            const uint64_t units = static_cast<uint64_t>(batch) * n_kv_heads * ((seq + 31) / 32);
            const unsigned grid = static_cast<unsigned>(spread_ctas(static_cast<int64_t>(units), di.sms));
            return launch_overlapped(kernel, grid, spread_threads(static_cast<int64_t>(units), static_cast<int>(grid), kMmaWarps), kSmemCtaBytes, s, static_cast<const uint8_t*>(d_meta),
                                     d_kblocks, batch * n_kv_heads, seq, q_per_kv, static_cast<const __half*>(d_q), scale, d_scores);
        }
    }
}

// ---------------------------------------------------------------------------------------------
// ecco_attn_values
// ---------------------------------------------------------------------------------------------
namespace {
// Warps of a CTA of ecco_attn_values that decode.  20 find room (9.4 KB of shared memory per warp), but with more than 16 a thread has 96
// registers and the kernel spills a little and takes a few percent more per tile: two kernels, and units of 17 to 19 tiles only where
// they save turns (a [16][8][32768][128] cache, eight heads, 534 us with 16 and 518 with 19; [8][32][4096][128] 162 and 166, by an earlier
// state of the kernel).  20, which takes the same registers, has not been measured.
constexpr int kAvWarps = 16, kAvManyWarps = 19;
struct AvPlan { int grid, unit_warps, teams; size_t partial_bytes, ticket_bytes; };
// How a CTA's warps share the work.  A unit is unit_warps tiles (of 32 tokens) of one head.
// One team: the units of all heads are split evenly over the CTAs, and all SMs should be busy for the same number of turns.  A turn
// costs about the time of six tiles' decoding however few tiles it has (6, 16 and 40 measured alike), so long rows take the
// largest units (16 x 8 x 32768 tokens: 19 warps) and short ones are cut until every SM has some.  Against 16 warps throughout:
// 8 x 32 x 64 tokens 27.1 -> 22.2 us, 2 x 8 x 777 17.4 -> 15.9, 1 x 1 x 32768 39.9 -> 25.5.
// Several teams of warps, each with heads of its own, for many short rows: one team spends 5 us on every head's reduction, most of it
// waiting, and the warps beyond the row's few tiles have nothing to do.  Against one team: 32 x 32 x 40 tokens 69.7 -> 17.6 us, 8 x 32 x 64
// 22.2 -> 14.4, 16 x 32 x 300 48.8 -> 34.5, 32 x 8 x 700 49.9 -> 33.9; from 4 x 32 x 1500 on one team is as fast (49.2 against 50.0).
void av_teams(AvPlan* p, int heads, int seq)
{
    constexpr int64_t kTurn = 6, kReduce = 10;             // a turn's fixed cost, and that of the reduction of a head, in tiles' decoding
    const int64_t tiles = (seq + 31) / 32, ctas = p->grid;
    int64_t best = INT64_MAX;
    p->teams = 1;
    for (int w = kAvManyWarps; w >= 1; --w) {
        const int64_t units = heads * ((tiles + w - 1) / w), turns = (units + ctas - 1) / ctas;
        int64_t cost = turns * (kTurn + w) + std::max<int64_t>(1, (heads + ctas - 1) / ctas - 1) * kReduce;
        if (w > kAvWarps) cost += cost / 32 + 1;
        if (cost < best) { best = cost; p->unit_warps = w; }
    }
    for (int t = 2; t <= kAvWarps; ++t) {
        const int64_t per_team = (heads + ctas * t - 1) / (ctas * t), active = std::min<int64_t>(t, (heads + ctas - 1) / ctas);
        for (int w = 1; w * t <= kAvWarps; ++w) {
            const int64_t cost = per_team * ((tiles + w - 1) / w * (kTurn + w * active) + kReduce);
            if (cost < best) { best = cost; p->unit_warps = w; p->teams = t; }
        }
    }
}
AvPlan av_plan(int batch, int n_kv_heads, int seq, int ctas_max)
{
    AvPlan p;
    const int heads = batch * n_kv_heads;
    // at most this many units; the device splits what there is evenly
    p.grid = spread_ctas(static_cast<int64_t>(heads) * ((seq + 31) / 32), ctas_max);
    av_teams(&p, heads, seq);
    auto up = [](size_t v) { return (v + 255) & ~static_cast<size_t>(255); };
    p.partial_bytes = up(static_cast<size_t>(p.grid + heads) * kPieceFloats * sizeof(float));
    p.ticket_bytes = up(static_cast<size_t>(heads) * sizeof(Ticket));
    return p;
}

template <int kWarps, bool kGiveUp = false>
int launch_attn_values(const DeviceInfo& di, const AvPlan& p, const void* d_meta, const uint8_t* d_vblocks, int heads, int seq,
                       int q_per_kv, const float* d_scores, float* d_out, float* partial, Ticket* tickets, cudaStream_t s)
{
    auto kernel = ecco_attn_values_kernel<kWarps, kGiveUp>;
    static thread_local bool configured[64] = {};
    const int rc = want_all_smem(kernel, &configured[di.device]);
    if (rc) return rc;
    // at least eight warps: those beyond the unit's help with the reductions
    const int warps = p.unit_warps * p.teams < 8 ? 8 : p.unit_warps * p.teams;
    return launch_overlapped(kernel, static_cast<unsigned>(p.grid), static_cast<unsigned>(warps * 32), kSmemCtaBytes, s,
                             static_cast<const uint8_t*>(d_meta), d_vblocks, heads, seq, q_per_kv, p.unit_warps, p.teams, d_scores, d_out, partial, tickets, next_ticket_tag());
}
}  // namespace

extern "C" size_t ecco_attn_values_workspace_bytes(int32_t batch, int32_t n_kv_heads, int32_t seq, int32_t q_per_kv)
{
    if (batch <= 0 || n_kv_heads <= 0 || seq <= 0 || q_per_kv < 1 || q_per_kv > 8) return 0;
    if (static_cast<int64_t>(batch) * n_kv_heads > (1 << 24)) return 0;
    const AvPlan p = av_plan(batch, n_kv_heads, seq, 256);
    return p.partial_bytes + p.ticket_bytes;
}

template <bool kGiveUp>
static int attn_values(const void* d_meta, const uint8_t* d_vblocks, int32_t batch, int32_t n_kv_heads, int32_t seq,
                       int32_t q_per_kv, const float* d_scores, float* d_out, void* d_workspace, size_t workspace_bytes,
                       void* stream)
{
    if (batch == 0 || n_kv_heads == 0) return (batch < 0 || n_kv_heads < 0) ? ECCO_ERR_INVALID_ARG : ECCO_OK;
    if (!d_meta || !d_vblocks || !d_scores || !d_out) return ECCO_ERR_INVALID_ARG;
    if (batch < 0 || n_kv_heads < 0 || seq <= 0 || q_per_kv < 1 || q_per_kv > 8) return ECCO_ERR_INVALID_ARG;
    if (static_cast<int64_t>(batch) * n_kv_heads > (1 << 24)) return ECCO_ERR_INVALID_ARG;
    if (!aligned16(d_meta) || !aligned16(d_vblocks) || !aligned16(d_scores) || !aligned16(d_out)) return ECCO_ERR_ALIGNMENT;
    DeviceInfo di;
    int rc = device_info(&di);
    if (rc) return rc;
    const AvPlan p = av_plan(batch, n_kv_heads, seq, di.sms < 256 ? di.sms : 256);
    if (!d_workspace || !aligned16(d_workspace)) return d_workspace ? ECCO_ERR_ALIGNMENT : ECCO_ERR_WORKSPACE;
    if (workspace_bytes < p.partial_bytes + p.ticket_bytes) return ECCO_ERR_WORKSPACE;
    if (kGiveUp && p.unit_warps > kAvWarps) return ECCO_ERR_INVALID_ARG;       // no kernel for it
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    uint8_t* wsb = static_cast<uint8_t*>(d_workspace);
    float* partial = reinterpret_cast<float*>(wsb);
    Ticket* tickets = reinterpret_cast<Ticket*>(wsb + p.partial_bytes);
    auto launch = p.unit_warps > kAvWarps ? launch_attn_values<kAvManyWarps> : launch_attn_values<kAvWarps, kGiveUp>;
    return launch(di, p, d_meta, d_vblocks, batch * n_kv_heads, seq, q_per_kv, d_scores, d_out, partial, tickets, s);
}

extern "C" int ecco_attn_values(const void* d_meta, const uint8_t* d_vblocks, int32_t batch, int32_t n_kv_heads, int32_t seq,
                                int32_t q_per_kv, const float* d_scores, float* d_out, void* d_workspace, size_t workspace_bytes,
                                void* stream)
{
    return attn_values<false>(d_meta, d_vblocks, batch, n_kv_heads, seq, q_per_kv, d_scores, d_out, d_workspace, workspace_bytes, stream);
}

extern "C" int ecco_test_attn_values_give_up(const void* d_meta, const uint8_t* d_vblocks, int32_t batch, int32_t n_kv_heads, int32_t seq,
                                             int32_t q_per_kv, const float* d_scores, float* d_out, void* d_workspace, size_t workspace_bytes,
                                             void* stream)
{
    return attn_values<true>(d_meta, d_vblocks, batch, n_kv_heads, seq, q_per_kv, d_scores, d_out, d_workspace, workspace_bytes, stream);
}


extern "C" int ecco_act_decompress(const uint8_t* d_blocks, uint64_t n_groups, void* d_out_fp16, void* stream)
{
    if (n_groups == 0) return ECCO_OK;
    if (!d_blocks || !d_out_fp16) return ECCO_ERR_INVALID_ARG;
    if (!aligned16(d_blocks) || (reinterpret_cast<uintptr_t>(d_out_fp16) & 31u)) return ECCO_ERR_ALIGNMENT;
    if (n_groups > kMaxGroups) return ECCO_ERR_INVALID_ARG;
    DeviceInfo di;
    int rc = device_info(&di);
    if (rc) return rc;
    const uint64_t n_chunks = n_groups * 4;
    return launch_overlapped(ecco_act_decompress_kernel, act_ctas(n_chunks, 1), static_cast<unsigned>(kActThreads), 0, static_cast<cudaStream_t>(stream),
                             reinterpret_cast<const uint4*>(d_blocks), n_chunks, static_cast<uint4*>(d_out_fp16));
}

extern "C" int ecco_act_compress(const void* d_x_fp16, uint64_t n_groups, uint8_t* d_blocks, void* stream)
{
    if (n_groups == 0) return ECCO_OK;
    if (!d_blocks || !d_x_fp16) return ECCO_ERR_INVALID_ARG;
    if (!aligned16(d_blocks) || (reinterpret_cast<uintptr_t>(d_x_fp16) & 31u)) return ECCO_ERR_ALIGNMENT;
    if (n_groups > kMaxGroups) return ECCO_ERR_INVALID_ARG;
    DeviceInfo di;
    int rc = device_info(&di);
    if (rc) return rc;
    const uint64_t n_chunks = n_groups * 4;
    const int loads = act_compress_loads(n_chunks, di);
    return launch_overlapped(loads == 1 ? ecco_act_compress_kernel<1> : ecco_act_compress_kernel<2>, act_ctas(n_chunks, loads), static_cast<unsigned>(kActThreads), 0,
                             static_cast<cudaStream_t>(stream), static_cast<const uint4*>(d_x_fp16), n_chunks, reinterpret_cast<uint4*>(d_blocks));
}


// calls of at least this many groups: eight lanes per group and tables in shared memory (see the kernel)
constexpr uint64_t kKvManyGroups = 16384;

// kinds: tensors of n_groups groups each that share the CTAs
template <class Groups>
static int launch_kv_compress(const DeviceInfo& di, const Groups& groups, uint64_t n_groups, int kinds, cudaStream_t s)
{
    if (!Groups::kFewToo || n_groups * kinds >= kKvManyGroups) {
        static thread_local bool configured[64] = {};
        if (!configured[di.device]) {
            const int rc = set_smem(ecco_kv_compress_many_kernel<Groups>, sizeof(KvManySmem));
            if (rc) return rc;
            configured[di.device] = true;
        }
        return launch_overlapped(ecco_kv_compress_many_kernel<Groups>, static_cast<unsigned>(kinds * spread_ctas(static_cast<int64_t>((n_groups + 3) / 4), di.sms / kinds)),
                                 static_cast<unsigned>(kKvManyWarps * 32), sizeof(KvManySmem), s, groups, n_groups);
    }
    if constexpr (Groups::kFewToo) {
        const uint64_t ctas = (n_groups + kKvWarps - 1) / kKvWarps;
        const uint64_t cap = static_cast<uint64_t>(di.sms) * 8 / kinds;
        return launch_overlapped(ecco_kv_compress_kernel<Groups>, static_cast<unsigned>(kinds * (ctas < cap ? ctas : cap)), static_cast<unsigned>(kKvWarps * 32), 0, s, groups,
                                 n_groups);
    }
}

extern "C" int ecco_kv_compress(const void* d_meta, const void* d_x_fp16, uint64_t n_groups, uint8_t* d_blocks, void* stream)
{
    if (n_groups == 0) return ECCO_OK;
    if (!d_meta || !d_x_fp16 || !d_blocks) return ECCO_ERR_INVALID_ARG;
    if (!aligned16(d_meta) || !aligned16(d_x_fp16) || !aligned16(d_blocks)) return ECCO_ERR_ALIGNMENT;
    if (n_groups > kMaxGroups) return ECCO_ERR_INVALID_ARG;
    DeviceInfo di;
    int rc = device_info(&di);
    if (rc) return rc;
    const DenseGroups groups = {static_cast<const uint8_t*>(d_meta), static_cast<const __half*>(d_x_fp16), d_blocks};
    return launch_kv_compress(di, groups, n_groups, 1, static_cast<cudaStream_t>(stream));
}

// ---------------------------------------------------------------------------------------------
// Paged KV cache
// ---------------------------------------------------------------------------------------------
static bool aligned_to(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
// log2 of the page size, or -1
static int page_shift_of(int32_t page_size)
{
    for (int sh = 0; sh <= 12; ++sh)
        if (page_size == 1 << sh) return sh;
    return -1;
}
static int check_paged_cache(const ecco_paged_cache* c)
{
    if (!c || !c->d_k_meta || !c->d_v_meta || !c->d_k_blocks || !c->d_v_blocks) return ECCO_ERR_INVALID_ARG;
    if (c->n_pages < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 65535 || page_shift_of(c->page_size) < 0) return ECCO_ERR_INVALID_ARG;
    if (static_cast<int64_t>(c->n_pages) * c->page_size > INT32_MAX) return ECCO_ERR_INVALID_ARG;
    if (!aligned16(c->d_k_meta) || !aligned16(c->d_v_meta) || !aligned_to(c->d_k_blocks, 32) || !aligned_to(c->d_v_blocks, 32)) return ECCO_ERR_ALIGNMENT;
    return ECCO_OK;
}

extern "C" int ecco_paged_plan(int32_t page_size, int32_t n_pages, int32_t n_req, const int32_t* d_ctx_lens, const int32_t* d_new_lens,
                               const int32_t* d_free_pages, int32_t n_free, int32_t* d_block_tables, int32_t table_stride, int32_t* d_slots,
                               int32_t n_slots, int32_t* d_cu_new, int32_t* d_kv_lens, int32_t* d_kv_tiles, int32_t* d_result, void* stream)
{
    const int shift = page_shift_of(page_size);
    if (shift < 0 || n_pages < 1 || static_cast<int64_t>(n_pages) * page_size > INT32_MAX) return ECCO_ERR_INVALID_ARG;
    if (n_req < 0 || n_req > 65535 || n_free < 0 || table_stride < 0 || n_slots < 0) return ECCO_ERR_INVALID_ARG;
    if (!d_cu_new || !d_kv_tiles || !d_result || (n_slots && !d_slots) || (n_free && !d_free_pages)) return ECCO_ERR_INVALID_ARG;
    if (n_req && (!d_ctx_lens || !d_new_lens || !d_kv_lens || (table_stride && !d_block_tables))) return ECCO_ERR_INVALID_ARG;
    for (const void* p : {static_cast<const void*>(d_ctx_lens), static_cast<const void*>(d_new_lens), static_cast<const void*>(d_free_pages),
                          static_cast<const void*>(d_block_tables), static_cast<const void*>(d_slots), static_cast<const void*>(d_cu_new),
                          static_cast<const void*>(d_kv_lens), static_cast<const void*>(d_kv_tiles), static_cast<const void*>(d_result)})
        if (!aligned_to(p, 4)) return ECCO_ERR_ALIGNMENT;
    // in place it cannot be done: every CTA reads all lengths, whatever the others have written
    if (n_req && (d_kv_lens == d_ctx_lens || d_kv_lens == d_new_lens)) return ECCO_ERR_INVALID_ARG;
    DeviceInfo di;
    const int rc = device_info(&di);
    if (rc) return rc;
    PagedPlan p = {};
    p.ctx = d_ctx_lens; p.added = d_new_lens; p.free_pages = d_free_pages;
    p.tables = d_block_tables; p.slots = d_slots; p.cu_new = d_cu_new; p.kv_lens = d_kv_lens; p.kv_tiles = d_kv_tiles; p.result = d_result;
    p.page_shift = shift; p.n_pages = n_pages; p.n_req = n_req; p.n_free = n_free; p.stride = table_stride; p.n_slots = n_slots;
    const int ctas = spread_ctas((static_cast<int64_t>(n_slots) + kPlanThreads - 1) / kPlanThreads, di.sms);
    return launch_overlapped(ecco_paged_plan_kernel, static_cast<unsigned>(ctas > 0 ? ctas : 1), static_cast<unsigned>(kPlanThreads), 0,
                             static_cast<cudaStream_t>(stream), p);
}

// Groups (of K, and as many of V) from which on K and V are compressed one after the other, each by all CTAs: they rarely take equally long, and
// half of the CTAs would wait for the others; below, the second launch costs more.  One launch / two, in us: 48 000 groups 61 / 64,
// 65 536 groups 72 / 77 (74 / 77 of 32 heads), 88 000 groups 96 / 91, 96 000 groups 98 / 99, 109 000 groups 113 / 105, 131 072 groups 125 / 118.
constexpr uint64_t kAppendTwoGroups = 81920;
static_assert(kAppendTwoGroups >= kKvManyGroups, "K or V alone is always a call of many groups");
extern "C" int ecco_paged_append(const ecco_paged_cache* cache, const void* d_k, const void* d_v, int64_t token_stride, const int32_t* d_slots,
                                 int32_t n_tokens, void* stream)
{
    int rc = check_paged_cache(cache);
    if (rc) return rc;
    if (n_tokens < 0) return ECCO_ERR_INVALID_ARG;
    if (n_tokens == 0) return ECCO_OK;
    if (!d_k || !d_v || !d_slots || token_stride < static_cast<int64_t>(cache->n_kv_heads) * kGroup) return ECCO_ERR_INVALID_ARG;
    if (!aligned16(d_k) || !aligned16(d_v) || token_stride % 8 || !aligned_to(d_slots, 4)) return ECCO_ERR_ALIGNMENT;
    DeviceInfo di;
    rc = device_info(&di);
    if (rc) return rc;
    const uint64_t n_groups = static_cast<uint64_t>(n_tokens) * cache->n_kv_heads;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    auto launch = [&](auto g, int kinds) {
        g.k_image = static_cast<const uint8_t*>(cache->d_k_meta); g.v_image = static_cast<const uint8_t*>(cache->d_v_meta);
        g.k = static_cast<const __half*>(d_k); g.v = static_cast<const __half*>(d_v);
        g.k_blocks = cache->d_k_blocks; g.v_blocks = cache->d_v_blocks;
        g.slots = d_slots; g.token_stride = token_stride;
        g.heads = cache->n_kv_heads; g.page_shift = page_shift_of(cache->page_size); g.n_slots = cache->n_pages * cache->page_size;
        g.inverse = static_cast<uint32_t>(std::min<uint64_t>((1ull << 32) / static_cast<uint64_t>(g.heads), UINT32_MAX));
        return launch_kv_compress(di, g, n_groups, kinds, s);
    };
    if (n_groups < kAppendTwoGroups) return launch(PagedGroups<2>{}, 2);
    rc = launch(PagedGroups<0>{}, 1);
    return rc ? rc : launch(PagedGroups<1>{}, 1);
}

namespace {
constexpr float kLog2E = 1.4426950408889634f;
// Tiles per warp (of each kind) from which on every CTA decodes both kinds, which costs a second set of tables and saves the wait of those
// CTAs whose kind is done first (8 requests of five rows, 8 heads, halves / both, in us: 1.0 tiles 90 / 97, 2.0 tiles 129 / 129, 3.0 tiles 167 / 170,
// 4.0 tiles 207 / 205, 4.6 tiles 229 / 232, 5.0 tiles 248 / 244, 5.6 tiles 265 / 268, 6.0 tiles 284 / 277, 10 tiles 437 / 419), and from
// which on one or two rows to a request take the products with K at once (8 requests of 1600 tokens, 32 heads, 2.8 tiles: 118 -> 106 us;
// of 1024, 1.8 tiles: 80 -> 75; of 800, 1.4 tiles: 67 -> 66).  With three to eight rows that pays later: 8 requests, 8 heads, three / eight
// rows, 2.1 tiles: 99 / 101 -> 103 / 106; 4.1 tiles: 163 / 167 -> 164 / 170; 6.1 tiles: 234 / 234 -> 225 / 234; 13.6 tiles: 530 / 531 -> 506 / 520.
constexpr int kStageBothTiles = 5, kScoresTiles = 1, kScoresMmaTiles = 6;
// Workspace of a launch over some KV heads, all offsets multiples of 256:
//   tiles | schedule: few_tiles, block_tiles, blocks, n_blocks, tickets, cuts | few rows: sums, maxima | many rows: sums, maxima
struct PagedAttnPlan {
    bool many;                         // there may be requests of more than kFewRows rows
    int few_ctas, many_ctas, max_blocks;
    size_t few_tiles, block_tiles, blocks, n_blocks, tickets, cuts, few_part, few_ml, many_part, many_ml, bytes;
};
PagedAttnPlan paged_attn_plan(const ecco_paged_batch& b, int heads, int q_per_kv, int ctas_max)
{
    PagedAttnPlan p = {};
    const int64_t rows = static_cast<int64_t>(b.max_new) * q_per_kv;
    p.many = rows > kFewRows;
    p.few_ctas = std::max(1, spread_ctas(static_cast<int64_t>(b.max_tiles) * heads, ctas_max));
    p.many_ctas = ctas_max;
    p.max_blocks = p.many ? b.n_tokens / (2 * tile_rows_tokens(q_per_kv)) + std::min(b.n_req, b.n_tokens) + 1 : 0;
    size_t at = static_cast<size_t>(std::max(b.max_tiles, 1)) * heads * 2 * kKvTileBytes;          // one at least: the tensor map has to have some
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at = (at + bytes + 255) & ~static_cast<size_t>(255);
        return here;
    };
    static_assert(kFewWarps<true> >= kFewWarps<false>, "places for either");
    const size_t few_slots = static_cast<size_t>(p.few_ctas) * kFewWarps<true> * 2 * kFewRows;
    const size_t many_slots = p.many ? static_cast<size_t>(p.many_ctas) * 2 * kManyRows : 0;
    p.few_tiles = take((static_cast<size_t>(b.n_req) + 1) * 4);
    p.block_tiles = take((static_cast<size_t>(p.max_blocks) + 1) * 4);
    p.blocks = take(static_cast<size_t>(p.max_blocks) * 8);
    p.n_blocks = take(8);                                  // and the number of rows to join
    p.tickets = take(static_cast<size_t>(2) * p.many_ctas * 4);
    p.cuts = take(static_cast<size_t>(p.few_ctas) * kFewWarps<true> * kFewRows * sizeof(FewCut));
    p.few_part = take(few_slots * kGroup * sizeof(float));
    p.few_ml = take(few_slots * sizeof(float2));
    p.many_part = take(many_slots * kGroup * sizeof(float));
    p.many_ml = take(many_slots * sizeof(float2));
    p.bytes = at;
    return p;
}
bool paged_batch_fine(const ecco_paged_cache& c, const ecco_paged_batch& b, int q_per_kv)
{
    if (b.n_req < 0 || b.n_req > 65535 || b.n_tokens < 0 || b.table_stride < 0 || b.max_new < 0 || b.max_kv < 0 || b.max_tiles < 0) return false;
    if (q_per_kv < 1 || q_per_kv > 16 || static_cast<int64_t>(c.n_kv_heads) * q_per_kv > 65535) return false;
    if (static_cast<int64_t>(b.max_tiles) * c.n_kv_heads > INT32_MAX / 2 || static_cast<int64_t>(b.max_tiles) > INT32_MAX / 32) return false;
    if (static_cast<int64_t>(b.n_tokens) * c.n_kv_heads * q_per_kv > INT32_MAX - 1024) return false;
    // tiles of all blocks of rows together are counted in 32 bits
    const int64_t blocks = static_cast<int64_t>(b.n_tokens) / (2 * tile_rows_tokens(q_per_kv)) + b.n_req + 1;
    return blocks * (static_cast<int64_t>(b.max_kv) / kManyTokens + 1) <= INT32_MAX;
}

// the tiles of a workspace as [piece][tile][1 KB]: a box of eight pieces of four tiles is a K or V operand of 128 tokens
bool make_tile_map(CUtensorMap* map, const PagedKv& kv)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {kPieceBytes / 4, static_cast<cuuint64_t>(2) * kv.heads * kv.max_tiles, 8};
    const cuuint64_t strides[2] = {kKvTileBytes, kPieceBytes};
    const cuuint32_t box[3] = {kPieceBytes / 4, kManyTokens / 32, 8};
    const cuuint32_t unit[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, kv.staged, dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// q as [token][query head][dim]: a box is sixteen dims of a tile of rows, as an operand has them
bool make_q_map(CUtensorMap* map, const PagedKv& kv, const PagedOut& o)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {kGroup, static_cast<cuuint64_t>(o.q_heads), static_cast<cuuint64_t>(kv.n_tokens)};
    const cuuint64_t strides[2] = {kGroup * 2, static_cast<cuuint64_t>(o.q_stride) * 2};
    const cuuint32_t box[3] = {16, static_cast<cuuint32_t>(o.q_per_kv), static_cast<cuuint32_t>(tile_rows_tokens(o.q_per_kv))};
    const cuuint32_t unit[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, const_cast<__half*>(o.q), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_32B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// k_map, v_map: as the kernel has them
template <bool k8>
int launch_paged_many(const DeviceInfo& di, const PagedKv& kv, const PagedOut& o, const PagedSchedule& sc, int ctas, const CUtensorMap& k_map, const CUtensorMap& v_map, cudaStream_t s)
{
    CUtensorMap q_map;
    if (!make_q_map(&q_map, kv, o)) return ECCO_ERR_CUDA;
    static thread_local bool configured[64] = {};
    if (!configured[di.device]) {
        const int rc = set_smem(ecco_paged_many_kernel<k8>, ManyShape<k8>::kBytes);
        if (rc) return rc;
        configured[di.device] = true;
    }
    return launch_overlapped(ecco_paged_many_kernel<k8>, static_cast<unsigned>(ctas), static_cast<unsigned>(ManyShape<k8>::kThreads), ManyShape<k8>::kBytes, s, kv, o, sc, k_map, v_map, q_map);
}
template <bool kScores>
int launch_paged_few(const DeviceInfo& di, const PagedKv& kv, const PagedOut& o, const PagedSchedule& sc, const PagedAttnPlan& p, cudaStream_t s)
{
    static thread_local bool configured[64] = {};
    if (!configured[di.device]) {
        const int rc = set_smem(ecco_paged_few_kernel<kScores>, kFewSmemBytes<kScores>);
        if (rc) return rc;
        configured[di.device] = true;
    }
    const int rc = launch_overlapped(ecco_paged_few_kernel<kScores>, static_cast<unsigned>(p.few_ctas), static_cast<unsigned>(kFewWarps<kScores> * 32), kFewSmemBytes<kScores>, s, kv, o, sc);
    if (rc) return rc;
    return launch_overlapped(ecco_paged_join_kernel, static_cast<unsigned>(std::min(p.few_ctas * kFewWarps<kScores>, di.sms * kJoinCtas)), 256u, 0, s, o);
}
template <StageKind kKind>
int launch_paged_stage(const DeviceInfo& di, const PagedKv& kv, const PagedOut& o, const PagedSchedule& sc, int64_t units, cudaStream_t s)
{
    static thread_local bool configured[64] = {};
    auto kernel = ecco_paged_stage_kernel<32, kKind>;
    int rc = want_all_smem(kernel, &configured[di.device]);
    if (rc) return rc;
    const int ctas = std::max(1, spread_ctas(units, kKind == kHalves ? di.sms / 2 : di.sms));
    return launch_overlapped(kernel, static_cast<unsigned>(kKind == kHalves ? 2 * ctas : ctas), spread_threads(units, ctas, 32), kSmemCtaBytes, s, kv, o, sc);
}
template <int kV>
int launch_paged_scores(const DeviceInfo& di, const PagedKv& kv, const PagedOut& o, float* scores, int64_t units, cudaStream_t s)
{
    static thread_local bool configured[64] = {};
    auto kernel = ecco_paged_scores_kernel<kV, fused_warps(kV)>;
    int rc = want_all_smem(kernel, &configured[di.device]);
    if (rc) return rc;
    const int ctas = std::max(1, spread_ctas(units, di.sms));
    return launch_overlapped(kernel, static_cast<unsigned>(ctas), spread_threads(units, ctas, fused_warps(kV)), kSmemCtaBytes, s, kv, o, scores);
}
int launch_paged_scores_mma(const DeviceInfo& di, const PagedKv& kv, const PagedOut& o, float* scores, int64_t units, cudaStream_t s)
{
    static thread_local bool configured[64] = {};
    auto kernel = ecco_paged_scores_mma_kernel<kMmaWarps>;
    int rc = want_all_smem(kernel, &configured[di.device]);
    if (rc) return rc;
    const int ctas = std::max(1, spread_ctas(units, di.sms));
    return launch_overlapped(kernel, static_cast<unsigned>(ctas), spread_threads(units, ctas, kMmaWarps), kSmemCtaBytes, s, kv, o, scores);
}
}  // namespace

extern "C" size_t ecco_paged_attn_workspace_bytes(const ecco_paged_cache* cache, const ecco_paged_batch* batch, int32_t q_per_kv)
{
    if (!cache || !batch || cache->n_kv_heads < 1 || cache->n_kv_heads > 65535 || !paged_batch_fine(*cache, *batch, q_per_kv)) return 0;
    return paged_attn_plan(*batch, cache->n_kv_heads, q_per_kv, 256).bytes;
}

extern "C" int ecco_paged_attn(const ecco_paged_cache* cache, const ecco_paged_batch* batch, int32_t q_per_kv, const void* d_q, int64_t q_stride,
                               float scale, uint32_t flags, void* d_out, float* d_lse, void* d_workspace, size_t workspace_bytes, void* stream)
{
    int rc = check_paged_cache(cache);
    if (rc) return rc;
    if (!batch || !paged_batch_fine(*cache, *batch, q_per_kv) || (flags & ~ECCO_ATTN_CAUSAL) || !std::isfinite(scale * kLog2E)) return ECCO_ERR_INVALID_ARG;
    const ecco_paged_batch& b = *batch;
    if (b.n_req == 0 || b.n_tokens == 0) return ECCO_OK;
    const int q_heads = cache->n_kv_heads * q_per_kv;
    if (!b.d_cu_new || !b.d_kv_lens || !b.d_kv_tiles || (b.table_stride && !b.d_block_tables) || !d_q || !d_out) return ECCO_ERR_INVALID_ARG;
    if (q_stride < static_cast<int64_t>(q_heads) * kGroup || q_stride >= 1ll << 38) return ECCO_ERR_INVALID_ARG;
    if (!aligned16(d_q) || q_stride % 8 || !aligned16(d_out) || !aligned_to(d_lse, 4)) return ECCO_ERR_ALIGNMENT;
    for (const int32_t* p : {b.d_block_tables, b.d_cu_new, b.d_kv_lens, b.d_kv_tiles})
        if (!aligned_to(p, 4)) return ECCO_ERR_ALIGNMENT;
    // in place it cannot be done: a row of q is read by whoever has tokens that it sees, at any time
    if (d_workspace && (d_out == d_q || d_out == d_workspace || d_q == d_workspace)) return ECCO_ERR_INVALID_ARG;
    DeviceInfo di;
    rc = device_info(&di);
    if (rc) return rc;
    if (!d_workspace || !aligned16(d_workspace)) return d_workspace ? ECCO_ERR_ALIGNMENT : ECCO_ERR_WORKSPACE;
    const int ctas = di.sms < 256 ? di.sms : 256;
    // as many heads at a time as the workspace holds
    int heads = cache->n_kv_heads;
    while (heads > 0 && paged_attn_plan(b, heads, q_per_kv, ctas).bytes > workspace_bytes) --heads;
    if (heads == 0) return ECCO_ERR_WORKSPACE;
    PagedKv kv = {};
    kv.k_meta = static_cast<const uint8_t*>(cache->d_k_meta); kv.v_meta = static_cast<const uint8_t*>(cache->d_v_meta);
    kv.k_blocks = cache->d_k_blocks; kv.v_blocks = cache->d_v_blocks;
    kv.tables = b.d_block_tables; kv.cu_new = b.d_cu_new; kv.kv_lens = b.d_kv_lens; kv.kv_tiles = b.d_kv_tiles;
    kv.n_pages = cache->n_pages; kv.page_shift = page_shift_of(cache->page_size); kv.all_heads = cache->n_kv_heads;
    kv.stride = b.table_stride; kv.n_req = b.n_req; kv.n_tokens = b.n_tokens; kv.max_tiles = std::max(b.max_tiles, 1);
    kv.max_new = b.max_new; kv.max_kv = b.max_kv;
    kv.staged = static_cast<uint8_t*>(d_workspace);
    PagedOut o = {};
    o.q = static_cast<const __half*>(d_q); o.q_stride = q_stride;
    o.scale_log2 = scale * kLog2E;
    o.q_per_kv = q_per_kv; o.q_heads = q_heads; o.causal = flags & ECCO_ATTN_CAUSAL;
    o.out = static_cast<__half*>(d_out); o.lse = d_lse;
    o.discard = aligned_to(d_workspace, 128);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    for (kv.head0 = 0; kv.head0 < cache->n_kv_heads; kv.head0 += kv.heads) {
        kv.heads = std::min(heads, cache->n_kv_heads - kv.head0);
        const PagedAttnPlan p = paged_attn_plan(b, kv.heads, q_per_kv, ctas);
        PagedSchedule sc = {};
        sc.few_tiles = reinterpret_cast<int32_t*>(kv.staged + p.few_tiles);
        sc.block_tiles = reinterpret_cast<int32_t*>(kv.staged + p.block_tiles);
        sc.blocks = reinterpret_cast<int2*>(kv.staged + p.blocks);
        sc.n_blocks = reinterpret_cast<int32_t*>(kv.staged + p.n_blocks);
        sc.n_cuts = sc.n_blocks + 1;
        sc.max_blocks = p.max_blocks;
        sc.few_rows = kFewRows;
        sc.tickets = reinterpret_cast<int32_t*>(kv.staged + p.tickets);
        sc.n_tickets = p.many ? 2 * p.many_ctas : 0;
        // Small calls decode K in half of the CTAs and V in the other half.  Large ones decode both in every CTA, or, for up to eight
        // rows to a request, take the products with K at once.
        const int64_t units = static_cast<int64_t>(b.max_tiles) * kv.heads;
        const int64_t per_warp = units / (31 * di.sms), rows = static_cast<int64_t>(b.max_new) * q_per_kv;
        const bool scores = rows >= 1 && rows <= kScoreRows && per_warp >= (rows <= 2 ? kScoresTiles : kScoresMmaTiles);
        if (scores) {
            // where K's tiles would be
            float* const at = reinterpret_cast<float*>(kv.staged + static_cast<size_t>(kv.heads) * kv.max_tiles * kKvTileBytes);
            o.scores = at;
            o.score_rows = static_cast<int32_t>(rows);
            rc = rows == 1   ? launch_paged_scores<1>(di, kv, o, at, units, s)
                 : rows == 2 ? launch_paged_scores<2>(di, kv, o, at, units, s)
                             : launch_paged_scores_mma(di, kv, o, at, units, s);
            if (!rc) rc = launch_paged_stage<kOnlyV>(di, kv, o, sc, units, s);
        } else {
            rc = per_warp >= kStageBothTiles ? launch_paged_stage<kBoth>(di, kv, o, sc, units, s) : launch_paged_stage<kHalves>(di, kv, o, sc, units, s);
        }
        if (rc) return rc;
        o.part = reinterpret_cast<float*>(kv.staged + p.few_part);
        o.part_ml = reinterpret_cast<float2*>(kv.staged + p.few_ml);
        o.cuts = reinterpret_cast<FewCut*>(kv.staged + p.cuts);
        o.n_cuts = sc.n_cuts;
        if (p.many) {
            PagedOut many = o;
            many.part = reinterpret_cast<float*>(kv.staged + p.many_part);
            many.part_ml = reinterpret_cast<float2*>(kv.staged + p.many_ml);
            CUtensorMap map;
            if (!make_tile_map(&map, kv)) return ECCO_ERR_CUDA;
            rc = launch_paged_many<false>(di, kv, many, sc, p.many_ctas, map, map, s);
            if (rc) return rc;
            o.early = 1;
        }
        rc = scores ? launch_paged_few<true>(di, kv, o, sc, p, s) : launch_paged_few<false>(di, kv, o, sc, p, s);
        if (rc) return rc;
    }
    return ECCO_OK;
}

// ---------------------------------------------------------------------------------------------
// Rotary positions
// ---------------------------------------------------------------------------------------------
static bool rope_fine(const ecco_rope* r)
{
    return r && r->rot_dim >= 16 && r->rot_dim <= kGroup && r->rot_dim % 16 == 0 && std::isfinite(r->gain) && !(r->flags & ~(ECCO_ROPE_NEIGHBOURS | ECCO_ROPE_INVERSE));
}

extern "C" int ecco_rope_apply(const ecco_rope* rope, const int32_t* d_positions, int32_t n_tokens, int32_t n_heads, const void* d_x, int64_t x_stride,
                               void* d_out, int64_t out_stride, void* stream)
{
    if (!rope_fine(rope) || n_tokens < 0 || n_heads < 1 || n_heads > 65535) return ECCO_ERR_INVALID_ARG;
    if (n_tokens == 0) return ECCO_OK;
    const int64_t row = static_cast<int64_t>(n_heads) * kGroup;
    if (!d_positions || !d_x || !d_out || x_stride < row || out_stride < row || x_stride >= 1ll << 38 || out_stride >= 1ll << 38) return ECCO_ERR_INVALID_ARG;
    if (!aligned16(d_x) || !aligned16(d_out) || x_stride % 8 || out_stride % 8 || !aligned_to(d_positions, 4)) return ECCO_ERR_ALIGNMENT;
    if (d_x == d_out && x_stride != out_stride) return ECCO_ERR_INVALID_ARG;       // rows over one another's
    DeviceInfo di;
    const int rc = device_info(&di);
    if (rc) return rc;
    RopeRows p = {};
    p.positions = d_positions;
    p.x = static_cast<const __half*>(d_x); p.out = static_cast<__half*>(d_out);
    p.x_stride = x_stride; p.out_stride = out_stride;
    p.n_tokens = n_tokens; p.n_heads = n_heads;
    // few tokens: their heads shared out, as far as every team of lanes has one
    const int64_t windows = (static_cast<int64_t>(n_tokens) + kRopeTokens - 1) / kRopeTokens;
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>((2 * di.sms + windows - 1) / windows, (n_heads + kRopeTeams - 1) / kRopeTeams));
    p.per_part = static_cast<int32_t>((n_heads + parts - 1) / parts);
    p.parts = (n_heads + p.per_part - 1) / p.per_part;
    return launch_overlapped(ecco_rope_kernel, static_cast<unsigned>(windows * p.parts), static_cast<unsigned>(kRopeThreads), 0, static_cast<cudaStream_t>(stream), *rope, p);
}

// ---------------------------------------------------------------------------------------------
// Paged KV cache in 8 bits
// ---------------------------------------------------------------------------------------------
static int check_paged8_cache(const ecco_paged8_cache* c)
{
    if (!c || !c->d_k || !c->d_v || !c->d_k_scales || !c->d_v_scales) return ECCO_ERR_INVALID_ARG;
    if (c->n_pages < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 65535 || page_shift_of(c->page_size) < 0) return ECCO_ERR_INVALID_ARG;
    if (static_cast<int64_t>(c->n_pages) * c->page_size > INT32_MAX) return ECCO_ERR_INVALID_ARG;
    if (!aligned16(c->d_k) || !aligned16(c->d_v) || !aligned_to(c->d_k_scales, 4) || !aligned_to(c->d_v_scales, 4)) return ECCO_ERR_ALIGNMENT;
    return ECCO_OK;
}

// rows of new tokens as [token][head][128]: a box is a run's
static bool make_rows_map(CUtensorMap* map, const P8Append& p, const __half* rows)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {kGroup, static_cast<cuuint64_t>(p.heads), static_cast<cuuint64_t>(p.n_tokens)};
    const cuuint64_t strides[2] = {kGroup * 2, static_cast<cuuint64_t>(p.token_stride) * 2};
    const cuuint32_t box[3] = {kGroup, 1, kP8Rows};
    const cuuint32_t unit[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, const_cast<__half*>(rows), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
template <bool kTurn>
static int launch_paged8_append(const DeviceInfo& di, const ecco_rope& rope, const P8Append& p, int64_t ctas, cudaStream_t s)
{
    static thread_local bool configured[64] = {};
    if (!configured[di.device]) {
        const int rc = set_smem(ecco_paged8_append_kernel<kTurn>, kP8AppendSmemBytes);
        if (rc) return rc;
        configured[di.device] = true;
    }
    CUtensorMap k_map, v_map;
    if (!make_rows_map(&k_map, p, p.k) || !make_rows_map(&v_map, p, p.v)) return ECCO_ERR_CUDA;
    return launch_overlapped(ecco_paged8_append_kernel<kTurn>, static_cast<unsigned>(ctas), static_cast<unsigned>(kP8AppendThreads), kP8AppendSmemBytes, s, rope, p, k_map, v_map);
}
extern "C" int ecco_paged8_append(const ecco_paged8_cache* cache, const ecco_rope* rope, const int32_t* d_positions, const void* d_k, const void* d_v,
                                  int64_t token_stride, const int32_t* d_slots, int32_t n_tokens, void* stream)
{
    int rc = check_paged8_cache(cache);
    if (rc) return rc;
    if (n_tokens < 0 || (rope && !rope_fine(rope))) return ECCO_ERR_INVALID_ARG;
    if (n_tokens == 0) return ECCO_OK;
    if (!d_k || !d_v || !d_slots || (rope && !d_positions) || token_stride < static_cast<int64_t>(cache->n_kv_heads) * kGroup || token_stride >= 1ll << 38) return ECCO_ERR_INVALID_ARG;
    if (!aligned16(d_k) || !aligned16(d_v) || token_stride % 8 || !aligned_to(d_slots, 4) || (rope && !aligned_to(d_positions, 4))) return ECCO_ERR_ALIGNMENT;
    DeviceInfo di;
    rc = device_info(&di);
    if (rc) return rc;
    P8Append p = {};
    p.positions = d_positions; p.slots = d_slots;
    p.k = static_cast<const __half*>(d_k); p.v = static_cast<const __half*>(d_v);
    p.k_codes = cache->d_k; p.v_codes = cache->d_v; p.k_scales = cache->d_k_scales; p.v_scales = cache->d_v_scales;
    p.token_stride = token_stride;
    p.n_tokens = n_tokens; p.n_slots = cache->n_pages * cache->page_size;
    p.heads = cache->n_kv_heads; p.page_shift = page_shift_of(cache->page_size);
    const int64_t windows = (static_cast<int64_t>(n_tokens) + kP8Rows - 1) / kP8Rows;
    // CTAs to a window, for three to an SM, of which two fit: finer shares even out windows that are not alike in work or fill the last round.  With two: single tokens cost less, prompts of
    // some hundred to a thousand rows more (three / two: 777 requests of one token, 32 heads 40.5 / 31.3 us, 8 heads 14.3 / 11.9; 256, 32 heads 17.2 / 14.7; but 1500, 32 heads
    // 77 / 84; prompts, 32 heads: 4 of 400 tokens 13.4 / 17.3, 8 of 300 22.4 / 32.7, 1 of 777 8.2 / 9.4; others alike), and the host does not know which it is.
    const int64_t slots = 3 * di.sms / windows;
    p.kinds = slots >= 2 ? 2 : 1;
    p.parts = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(slots / p.kinds, 2ll * p.heads)));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return rope ? launch_paged8_append<true>(di, *rope, p, windows * p.parts * p.kinds, s) : launch_paged8_append<false>(di, ecco_rope{}, p, windows * p.parts * p.kinds, s);
}

namespace {
// Rows of a request up to which they go to ecco_paged8_few_kernel, sixteen at a time; all rows do, where the tiles of the call, each once for sixteen rows, are few
constexpr int kP8FewRows = 64;
// (a request of 80 rows over 4000 tokens, 8 heads 59 -> 23 us, of 800 over 700 34.6 -> 29.2, over 200 24.5 -> 22.4; 16 000 tiles are as fast the other way).
constexpr int64_t kP8FewPasses = 10000;
// CTAs that a block's sums come from: a head of 800 rows over 16000 tokens from 126 / 32 / 16 CTAs 92 / 83 / 66 us, 8 heads of 320 rows over 4000 tokens from 9 / 8
// / 4 50 / 40 / 42
constexpr int kP8ManyJoins = 8;
// CTAs for few rows.  One to a request and head, so that no sums pass through memory, where there are at most as many and they have few tiles (2
// requests of 300 / 780 / 2000 tokens, 8 heads: 7.6 / 9.8 / 15.7 us, with equal parts of the line of four tiles or more 8.2 / 8.7 / 10.1), or where they fill the machine
// anyway (16 of 1500 to 2000 tokens, 8 heads 20.5 / 22.2).  Else equal parts, of four tiles at least (2 requests of 780, of two, four, eight: 9.8 / 8.7 / 11.0), and
// not so small that one request's sums come from more than 32 CTAs (one head of 16000 tokens, from 32, 64: 14.2 / 17.3).
constexpr int kP8OneCtaTiles = 16, kP8CtaTiles = 4, kP8JoinCtas = 32;
// Rows of a request from which on tiles of its pages in fp16 are made beforehand, if the workspace has room for them: every block of 256 rows reads
// them again.  Beforehand / in the kernel: 4 requests, 8 heads over 4096 tokens, 512 rows each 86 / 65 us, 1200 rows 137 / 141, 2308 rows 200 / 218; 2 of 8192
// rows 310 / 346; 8 of 4800 rows over 3000 tokens 511 / 639.
constexpr int64_t kP8StagedRows = 2304;
constexpr size_t kP8StagedMost = static_cast<size_t>(2) << 30;                   // more is not asked for
// Workspace, all offsets multiples of 256:
//   schedule | few rows: tickets, sums, maxima | many rows: sums, maxima | tiles, if any
struct P8AttnPlan {
    bool many, line, by_request;       // there may be requests of more rows; more requests than the kernel for few rows schedules itself
    int few_rows, few_ctas, many_ctas, max_blocks;
    size_t few_tiles, block_tiles, blocks, n_blocks, tickets, few_tickets, few_part, few_ml, many_part, many_ml, bytes;
    size_t tiles, bytes_with_tiles;    // the same as bytes where there are none
};
P8AttnPlan paged8_attn_plan(const ecco_paged_batch& b, int heads, int q_per_kv, int ctas_max)
{
    P8AttnPlan p = {};
    const int64_t rows = std::min<int64_t>(static_cast<int64_t>(b.max_new) * q_per_kv, INT32_MAX);      // a batch has no more, see paged_batch_fine
    const int64_t all_groups = (rows + kP8Rows16 - 1) / kP8Rows16, tiles = static_cast<int64_t>(b.max_tiles) * heads;
    p.few_rows = static_cast<int>(all_groups * tiles <= kP8FewPasses ? std::max<int64_t>(rows, kP8FewRows) : kP8FewRows);
    p.many = rows > p.few_rows;
    const bool room_for_many = rows > kP8FewRows;          // whatever max_tiles says
    p.line = b.n_req > kP8Reqs;
    const int64_t groups = std::min<int64_t>(all_groups, (p.few_rows + kP8Rows16 - 1) / kP8Rows16);
    const int64_t tiles_of_one = (static_cast<int64_t>(b.max_kv) + 31) / 32 * std::max<int64_t>(groups, 1), units = tiles * std::max<int64_t>(groups, 1);
    p.by_request = static_cast<int64_t>(b.n_req) * heads <= ctas_max && (tiles_of_one <= kP8OneCtaTiles || tiles_of_one * ctas_max * 3 <= units * 4);
    const int64_t per_cta = std::max<int64_t>(kP8CtaTiles, tiles_of_one / kP8JoinCtas);
    p.few_ctas = p.by_request ? std::max(b.n_req, 1) * heads : std::max(1, spread_ctas((units + per_cta - 1) / per_cta, ctas_max));
    // blocks' tiles of 128 tokens, at most; a block's sums come from some eight CTAs at most
    const int64_t many_units = (rows + kManyRows - 1) / kManyRows * ((tiles + 3) / 4), per_many = std::max<int64_t>(1, b.max_kv / (kManyTokens * kP8ManyJoins));
    p.many_ctas = static_cast<int>(std::min<int64_t>(ctas_max, std::max<int64_t>(1, many_units / per_many)));
    p.max_blocks = room_for_many ? b.n_tokens / (2 * tile_rows_tokens(q_per_kv)) + std::min(b.n_req, b.n_tokens) + 1 : 0;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at = (at + bytes + 255) & ~static_cast<size_t>(255);
        return here;
    };
    const size_t few_slots = static_cast<size_t>(ctas_max) * 2 * kP8Rows16, many_slots = room_for_many ? static_cast<size_t>(ctas_max) * 2 * kManyRows : 0;
    p.few_tiles = take((static_cast<size_t>(b.n_req) + 1) * 4);
    p.block_tiles = take((static_cast<size_t>(p.max_blocks) + 1) * 4);
    p.blocks = take(static_cast<size_t>(p.max_blocks) * 8);
    p.n_blocks = take(8);
    p.tickets = take(static_cast<size_t>(2) * ctas_max * 4);
    p.few_tickets = take(static_cast<size_t>(ctas_max) * kTicketStride * sizeof(Ticket));
    p.few_part = take(few_slots * kGroup * sizeof(float));
    p.few_ml = take(few_slots * sizeof(float2));
    p.many_part = take(many_slots * kGroup * sizeof(float));
    p.many_ml = take(many_slots * sizeof(float2));
    p.tiles = p.bytes = p.bytes_with_tiles = at;
    const size_t tile_bytes = static_cast<size_t>(tiles) * 2 * kKvTileBytes;
    if (p.many && rows > kP8StagedRows && tile_bytes <= kP8StagedMost) p.bytes_with_tiles = at + tile_bytes;
    return p;
}
// a pool as [page][head][place][128 bytes]: a box is a page's part of a tile of some tokens
bool make_p8_map(CUtensorMap* map, const PagedKv& kv, const uint8_t* pool, int tokens)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t page = 1ull << kv.page_shift;
    const cuuint64_t dims[4] = {kGroup, page, static_cast<cuuint64_t>(kv.all_heads), static_cast<cuuint64_t>(kv.n_pages)};
    const cuuint64_t strides[3] = {kGroup, kGroup * page, kGroup * page * kv.all_heads};
    const cuuint32_t box[4] = {kGroup, static_cast<cuuint32_t>(std::min<cuuint64_t>(page, static_cast<cuuint64_t>(tokens))), 1, 1};
    const cuuint32_t unit[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<uint8_t*>(pool), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// of K and of V, where the kernels use them
bool make_p8_maps(CUtensorMap* k_map, CUtensorMap* v_map, const PagedKv& kv, int tokens)
{
    return kv.page_shift < kP8SwizzledShift || (make_p8_map(k_map, kv, kv.k_blocks, tokens) && make_p8_map(v_map, kv, kv.v_blocks, tokens));
}
template <int kN>
int launch_paged8_few(const DeviceInfo& di, const PagedKv& kv, const PagedOut& o, const P8Few& f, int ctas, const CUtensorMap& k_map, const CUtensorMap& v_map, cudaStream_t s)
{
    static thread_local bool configured[64] = {};
    if (!configured[di.device]) {
        const int rc = set_smem(ecco_paged8_few_kernel<kN>, P8Smem<kN>::kBytes);
        if (rc) return rc;
        configured[di.device] = true;
    }
    return launch_overlapped(ecco_paged8_few_kernel<kN>, static_cast<unsigned>(ctas), static_cast<unsigned>(kP8Threads), P8Smem<kN>::kBytes, s, kv, o, f, k_map, v_map);
}
// the part of the batch's checks that ecco_paged_attn has: the pages are the same
bool paged8_batch_fine(const ecco_paged8_cache& c, const ecco_paged_batch& b, int q_per_kv)
{
    ecco_paged_cache same = {};
    same.n_kv_heads = c.n_kv_heads;
    return paged_batch_fine(same, b, q_per_kv);
}
}  // namespace

extern "C" size_t ecco_paged8_attn_workspace_bytes(const ecco_paged8_cache* cache, const ecco_paged_batch* batch, int32_t q_per_kv)
{
    if (!cache || !batch || cache->n_kv_heads < 1 || cache->n_kv_heads > 65535 || !paged8_batch_fine(*cache, *batch, q_per_kv)) return 0;
    return paged8_attn_plan(*batch, cache->n_kv_heads, q_per_kv, 256).bytes_with_tiles;
}

extern "C" int ecco_paged8_attn(const ecco_paged8_cache* cache, const ecco_paged_batch* batch, int32_t q_per_kv, const void* d_q, int64_t q_stride, float scale,
                                uint32_t flags, void* d_out, float* d_lse, void* d_workspace, size_t workspace_bytes, void* stream)
{
    int rc = check_paged8_cache(cache);
    if (rc) return rc;
    if (!batch || !paged8_batch_fine(*cache, *batch, q_per_kv) || (flags & ~ECCO_ATTN_CAUSAL) || !std::isfinite(scale * kLog2E)) return ECCO_ERR_INVALID_ARG;
    const ecco_paged_batch& b = *batch;
    if (b.n_req == 0 || b.n_tokens == 0) return ECCO_OK;
    const int q_heads = cache->n_kv_heads * q_per_kv;
    if (!b.d_cu_new || !b.d_kv_lens || !b.d_kv_tiles || (b.table_stride && !b.d_block_tables) || !d_q || !d_out) return ECCO_ERR_INVALID_ARG;
    if (q_stride < static_cast<int64_t>(q_heads) * kGroup || q_stride >= 1ll << 38) return ECCO_ERR_INVALID_ARG;
    if (!aligned16(d_q) || q_stride % 8 || !aligned16(d_out) || !aligned_to(d_lse, 4)) return ECCO_ERR_ALIGNMENT;
    for (const int32_t* p : {b.d_block_tables, b.d_cu_new, b.d_kv_lens, b.d_kv_tiles})
        if (!aligned_to(p, 4)) return ECCO_ERR_ALIGNMENT;
    // in place it cannot be done: a row of q is read by whoever has tokens that it sees, at any time
    if (d_workspace && (d_out == d_q || d_out == d_workspace || d_q == d_workspace)) return ECCO_ERR_INVALID_ARG;
    DeviceInfo di;
    rc = device_info(&di);
    if (rc) return rc;
    if (!d_workspace || !aligned16(d_workspace)) return d_workspace ? ECCO_ERR_ALIGNMENT : ECCO_ERR_WORKSPACE;
    const P8AttnPlan p = paged8_attn_plan(b, cache->n_kv_heads, q_per_kv, di.sms < 256 ? di.sms : 256);
    if (workspace_bytes < p.bytes) return ECCO_ERR_WORKSPACE;
    PagedKv kv = {};
    kv.k_meta = cache->d_k_scales; kv.v_meta = cache->d_v_scales;
    kv.k_blocks = cache->d_k; kv.v_blocks = cache->d_v;
    kv.tables = b.d_block_tables; kv.cu_new = b.d_cu_new; kv.kv_lens = b.d_kv_lens; kv.kv_tiles = b.d_kv_tiles;
    kv.n_pages = cache->n_pages; kv.page_shift = page_shift_of(cache->page_size); kv.all_heads = kv.heads = cache->n_kv_heads;
    kv.stride = b.table_stride; kv.n_req = b.n_req; kv.n_tokens = b.n_tokens; kv.max_tiles = std::max(b.max_tiles, 1);
    kv.max_new = b.max_new; kv.max_kv = b.max_kv;
    kv.staged = static_cast<uint8_t*>(d_workspace);
    PagedOut o = {};
    o.q = static_cast<const __half*>(d_q); o.q_stride = q_stride;
    o.scale_log2 = scale * kLog2E;
    o.q_per_kv = q_per_kv; o.q_heads = q_heads; o.causal = flags & ECCO_ATTN_CAUSAL;
    o.out = static_cast<__half*>(d_out); o.lse = d_lse;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    CUtensorMap k_map = {}, v_map = {};
    if (p.many || p.line) {
        PagedSchedule sc = {};
        sc.few_tiles = reinterpret_cast<int32_t*>(kv.staged + p.few_tiles);
        sc.block_tiles = reinterpret_cast<int32_t*>(kv.staged + p.block_tiles);
        sc.blocks = reinterpret_cast<int2*>(kv.staged + p.blocks);
        sc.n_blocks = reinterpret_cast<int32_t*>(kv.staged + p.n_blocks);
        sc.n_cuts = sc.n_blocks + 1;
        sc.max_blocks = p.max_blocks;
        sc.few_rows = p.few_rows;
        sc.tickets = reinterpret_cast<int32_t*>(kv.staged + p.tickets);
        sc.n_tickets = p.many ? 2 * p.many_ctas : 0;
        // they are written 32 bytes at a time
        const bool tiles = p.bytes_with_tiles > p.bytes && p.bytes_with_tiles <= workspace_bytes && aligned_to(d_workspace, 32);
        PagedKv staged = kv;
        staged.staged = kv.staged + p.tiles;
        const unsigned grid = tiles ? static_cast<unsigned>(spread_ctas(static_cast<int64_t>(b.max_tiles) * kv.heads / kP8StageWarps + 1, di.sms * 2)) : 1u;
        rc = launch_overlapped(ecco_paged8_stage_kernel, grid, tiles ? static_cast<unsigned>(kP8StageWarps * 32) : 32u, 0, s, staged, o, sc, static_cast<int32_t>(tiles),
                               static_cast<int32_t>(p.line));
        if (rc) return rc;
        if (p.many) {
            PagedOut many = o;
            many.part = reinterpret_cast<float*>(kv.staged + p.many_part);
            many.part_ml = reinterpret_cast<float2*>(kv.staged + p.many_ml);
            if (tiles) {
                CUtensorMap map;
                if (!make_tile_map(&map, staged)) return ECCO_ERR_CUDA;
                rc = launch_paged_many<false>(di, staged, many, sc, p.many_ctas, map, map, s);
            } else {
                if (!make_p8_maps(&k_map, &v_map, kv, kManyTokens)) return ECCO_ERR_CUDA;
                rc = launch_paged_many<true>(di, kv, many, sc, p.many_ctas, k_map, v_map, s);
            }
            if (rc) return rc;
            o.early = 1;
        }
    }
    if (!make_p8_maps(&k_map, &v_map, kv, 32)) return ECCO_ERR_CUDA;
    P8Few f = {};
    f.line = p.line ? reinterpret_cast<const int32_t*>(kv.staged + p.few_tiles) : nullptr;
    f.few_rows = p.few_rows;
    f.by_request = p.by_request;
    f.part = reinterpret_cast<float*>(kv.staged + p.few_part);
    f.part_ml = reinterpret_cast<float2*>(kv.staged + p.few_ml);
    f.tickets = reinterpret_cast<Ticket*>(kv.staged + p.few_tickets);
    f.tag = next_ticket_tag();
    return static_cast<int64_t>(b.max_new) * q_per_kv <= 8 ? launch_paged8_few<1>(di, kv, o, f, p.few_ctas, k_map, v_map, s) : launch_paged8_few<2>(di, kv, o, f, p.few_ctas, k_map, v_map, s);
}
