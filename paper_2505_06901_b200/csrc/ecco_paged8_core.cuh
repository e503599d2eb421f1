// ecco_paged8_core.cuh -- the format of the paged KV cache in 8 bits, and copies that its kernels share
// Part of the one translation unit ecco_kernels.cu; included from there only.
#pragma once

namespace {

// ---------------------------------------------------------------------------------------------
// The cache: E4M3 numbers, and a power of two 2^e for each block of min(16, page size) places of a page and head.  With e in -15 .. 7 every
// value is an fp16 number, so reading the cache rounds nothing; and a power of two that grows rounds only what becomes
// subnormal.
// ---------------------------------------------------------------------------------------------
constexpr int kP8Lowest = -15, kP8Highest = 7;
__device__ __forceinline__ int p8_exponent(uint32_t byte) { return min(max(static_cast<int>(byte) - 127, kP8Lowest), kP8Highest); }
// two E4M3 numbers of the lower / upper half of a word -> fp16, exactly
__device__ __forceinline__ uint32_t e4m3_low(uint32_t v)
{
    uint32_t r;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t}" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint32_t e4m3_high(uint32_t v)
{
    uint32_t r;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(r) : "r"(v));
    return r;
}
// four fp16 numbers -> E4M3, to nearest even, saturating
__device__ __forceinline__ uint32_t to_e4m3(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f16x2 l, %1;\n\tcvt.rn.satfinite.e4m3x2.f16x2 h, %2;\n\tmov.b32 %0, {l, h};\n\t}" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t mul_h2(uint32_t a, uint32_t b)
{
    const __half2 v = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&v);
}
// 2^n twice as fp16, n in -24 .. 15
__device__ __forceinline__ uint32_t power_h2(int n)
{
    const uint32_t h = n >= -14 ? static_cast<uint32_t>(n + 15) << 10 : 1u << (n + 24);
    return h | (h << 16);
}

__device__ __forceinline__ uint4 lds_v4(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}

__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
// more bytes to come before the barrier's phase is over, without an arrival
__device__ __forceinline__ void mbar_expect_more(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// a look that does not wait
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// The first n (1 .. 4) bytes of a word global -> shared, the others zero; the barrier counts an arrival of this thread's when all such copies that it has
// begun have come.  They go through L1 (copies past it have sixteen bytes, at addresses that scales need not have): only behind dependency_wait().
__device__ __forceinline__ void copy_word(uint32_t dst, const uint8_t* src, int n)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void arrive_with_words(uint32_t bar) { asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory"); }
// 3-D tiled bulk load global -> shared through a tensor map (TMA); what lies outside of the tensor reads as zero
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map), "r"(x),
                 "r"(y), "r"(z), "r"(bar)
                 : "memory");
}
// the same, 4-D
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z),
                 "r"(w), "r"(bar)
                 : "memory");
}
// Pages of eight tokens and more come through tensor maps that swap the 16-byte pieces of a row by its number mod 8, so that loads of several rows do not meet
// in a bank; smaller ones as they are.
constexpr int kP8SwizzledShift = 3;

}  // namespace
