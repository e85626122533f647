// What the kernels that multiply on the fifth-generation tensor cores share: bounded waits, scale words, tensor maps.
#pragma once
#include <cuda.h>

#include <atomic>

#include "zc_fp8.cuh"

namespace zc {

// What kernels of this file's user left behind (one word per translation unit).
static __device__ unsigned int g_fp8_timeout;
constexpr uint32_t kMarkGaveUp = 1, kMarkSettled = 2, kMarkUnsettled = 4;

// Every wait is bounded: on giving up the block is marked, and the other roles' waits end with it.  Blocks that copy into, or multiply
// from, each other's shared memory are marked together: `other` is the place of the other block's mark (0: there is none).
struct Waiter {
    uint32_t limit;
    volatile uint32_t* failed;
    uint32_t other = 0;
    template <bool CLUSTER = false>
    __device__ __forceinline__ bool operator()(uint32_t bar, uint32_t parity) const
    {
        for (uint32_t i = 0; i <= limit; ++i) {
            if (CLUSTER ? bar_try_cluster(bar, parity) : bar_try(bar, parity)) return true;
            if (*failed) return false;
        }
        give_up();
        return false;
    }
    __device__ __forceinline__ void give_up() const
    {
        *failed = 1;
        if (other) asm volatile("st.shared::cluster.u32 [%0], %1;" :: "r"(other), "r"(1u) : "memory");
    }
    // the same for all lanes of a converged warp at once
    __device__ __forceinline__ bool warp(uint32_t bar, uint32_t parity) const { return __all_sync(0xFFFFFFFFu, operator()(bar, parity)); }
    // for two barriers' phases
    __device__ __forceinline__ bool warp_both(uint32_t bar, uint32_t also, uint32_t parity) const
    {
        bool there = false;
        for (uint32_t i = 0; i <= limit; ++i) {
            there = bar_try(bar, parity) && bar_try(also, parity);
            if (there || *failed) break;
        }
        if (!there) give_up();
        return __all_sync(0xFFFFFFFFu, there);
    }
    __device__ __forceinline__ bool warp_across(uint32_t bar, uint32_t parity) const { return __all_sync(0xFFFFFFFFu, operator()<true>(bar, parity)); }
};

// Copies and matrix instructions that are under way read and write a block's shared and tensor memory, which the next block may get when
// this one ends, also when it gave up.  A block ends only once these have, or have been waited for as long as anything else: for phases
// that they alone complete, whatever other roles do.
__device__ __forceinline__ bool settled(uint32_t bar, uint32_t parity, uint32_t limit)
{
#pragma unroll 1
    for (uint32_t i = 0; i <= limit; ++i)
        if (bar_try(bar, parity)) return true;
    return false;
}
// The same for the stage that is a lane's, where `st` is the next one to be used, in round `round`.
__device__ __forceinline__ bool settled_stage(uint32_t first_bar, uint32_t lane, uint32_t stages, uint32_t st, uint32_t round, uint32_t limit)
{
    const uint32_t rounds = round + (lane < st);
    return lane >= stages || rounds == 0 || settled(first_bar + 8 * lane, (rounds - 1) & 1, limit);
}
// One thread of a block that gave up, when all of its roles have ended.
__device__ __forceinline__ void report(uint32_t unsettled) { atomicOr(&g_fp8_timeout, kMarkGaveUp | (unsettled ? kMarkUnsettled : kMarkSettled)); }

// The scale bytes of steps first .. first + 3 of one row as a word; 127 (a factor of 1) where there is none.
__device__ __forceinline__ uint32_t scale_word(const uint8_t* s, uint64_t ld, uint32_t square, uint32_t row, uint32_t rows, uint32_t first, uint32_t end)
{
    uint32_t w = 0x7F7F7F7Fu;
    if (row < rows) {
        const uint8_t* p = s + (uint64_t)(square ? row >> 7 : row) * ld + first;
        if (first + 4 <= end && (reinterpret_cast<uintptr_t>(p) & 3) == 0) return *reinterpret_cast<const uint32_t*>(p);
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            if (first + i < end) w = (w & ~(0xFFu << (8 * i))) | ((uint32_t)p[i] << (8 * i));
    }
    return w;
}

// ---- host ----

// The calling translation unit's word on the current device; null on an error.
static unsigned int* marks_word()
{
    void* p = nullptr;
    return cudaGetSymbolAddress(&p, g_fp8_timeout) == cudaSuccess ? (unsigned int*)p : nullptr;
}

// A number that is worked out on a device's first use (0: it failed, and is tried again), kept per device.
struct OncePerDevice {
    std::atomic<uint32_t> value[64] = {};
    template <typename F>
    uint32_t operator()(F work)
    {
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return work();
        uint32_t v = value[dev].load(std::memory_order_relaxed);
        if (!v) { v = work(); value[dev].store(v, std::memory_order_relaxed); }
        return v;
    }
};

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeFn encode_fn()
{
    static const EncodeFn fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) p = nullptr;
        return (EncodeFn)p;
    }();
    return fn;
}

// A matrix of bytes as tiles of `height` rows x 128 bytes in the 128-byte swizzle; what lies outside reads as zeros.
static bool make_map(CUtensorMap* map, const void* elems, uint64_t rows, uint64_t cols, uint64_t ld, uint32_t height)
{
    const cuuint64_t dims[2] = {cols, rows}, pitch[1] = {ld};
    const cuuint32_t box[2] = {128, height}, step[2] = {1, 1};
    return encode_fn() && encode_fn()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(elems), dims, pitch, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                      CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A matrix of results as pieces of 32 rows x 64 bytes in the 64-byte swizzle.
static bool make_result_map(CUtensorMap* map, void* out, uint32_t type, uint64_t rows, uint64_t cols, uint64_t ld_bytes)
{
    const cuuint64_t dims[2] = {cols, rows}, pitch[1] = {ld_bytes};
    const cuuint32_t box[2] = {64 / real_bytes(type), 32}, step[2] = {1, 1};
    const CUtensorMapDataType t = type == ZC_REAL_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : type == ZC_REAL_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    return encode_fn() && encode_fn()(map, t, 2, out, dims, pitch, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B,
                                      CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Descriptor of the scaled FP8 instruction without its scale selectors.
static uint32_t instruction_of(uint32_t format_a, uint32_t format_b, uint32_t m, uint32_t n)
{
    const uint32_t fa = format_a == ZC_FMT_FP8_E5M2, fb = format_b == ZC_FMT_FP8_E5M2;
    // A and B types, N / 8, E8M0 scales, M / 16; both operands have k as their fastest axis
    return (fa << 7) | (fb << 10) | ((n >> 3) << 17) | (1u << 23) | ((m >> 4) << 24);
}

}  // namespace zc
