// Writing a quantised key/value cache and reading it back.
//
// A thread has a block of 32 elements that share a scale byte: 64 bytes of BF16 in, 16 bytes of FP4 and one of scale out.  Nothing is read twice
// and threads need nothing of one another, so the memory's rate bounds it.  A thread block takes a few rows (tokens), all heads, keys and
// values; its threads go along a token's head first (what is side by side on both sides), then over the rows, which mostly are neighbours in a page.
#include <atomic>

#include "zc_kv.cuh"

namespace zc {

constexpr uint32_t kCacheThreads = 256, kCacheMaxRows = 16;

static __device__ unsigned int g_kv_marks;
constexpr uint32_t kKvAnswers = 1024;
static __device__ unsigned int g_kv_answers[kKvAnswers];
__global__ void kv_collect_kernel(unsigned int* marks, uint32_t at) { g_kv_answers[at] = atomicExch(marks, 0u); }

unsigned int* kv_marks_word()
{
    // looked up on a device's first use
    static std::atomic<unsigned int*> known[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return nullptr;
    const bool keep = dev >= 0 && dev < 64;
    if (keep)
        if (unsigned int* p = known[dev].load(std::memory_order_relaxed)) return p;
    void* p = nullptr;
    if (cudaGetSymbolAddress(&p, g_kv_marks) != cudaSuccess) return nullptr;
    if (keep) known[dev].store((unsigned int*)p, std::memory_order_relaxed);
    return (unsigned int*)p;
}

struct CacheParams {
    KvCache C;
    KvBatch B;
    KvTensor t[2];                    // keys, values
    uint32_t rows_per_block, sides;   // sides: 1 keys, 2 values, 3 both
};

// Where the block's rows lie: page * page_tokens + token of the page, -1 for no place, -2 for a row that is nobody's.
__device__ __forceinline__ void find_places(const CacheParams& P, int row0, int* places)
{
    if (threadIdx.x < 32) {
        const int found = kv_find(P.B, row0);
        const int row = row0 + (int)threadIdx.x;
        if (threadIdx.x < P.rows_per_block) {
            int place = -2, pos;
            uint32_t b = found < 0 ? 0 : (uint32_t)found;
            if (row < (int)P.B.n_rows && kv_position(P.B, row, b, pos)) {
                place = -1;
                if (pos >= 0) {
                    const int page = kv_page(P.C, P.B, b, (uint32_t)pos >> P.C.page_shift);
                    if (page >= 0) place = (page << P.C.page_shift) | (pos & ((1 << P.C.page_shift) - 1));
                }
            }
            places[threadIdx.x] = place;
        }
    }
}
// Number of a block's first element / 32 in the cache, for a place, a head, and `blocks` blocks a token's head.
__device__ __forceinline__ uint64_t block_at(const KvCache& C, int place, uint32_t head, uint32_t blocks, uint32_t blk)
{
    const uint32_t page = (uint32_t)place >> C.page_shift, token = (uint32_t)place & ((1u << C.page_shift) - 1);
    return ((((uint64_t)page * C.heads + head) << C.page_shift) + token) * blocks + blk;
}

// ---- 32 real numbers ----
template <typename T, bool WIDE>
__device__ __forceinline__ void load_block(const uint8_t* p, float v[32])
{
    constexpr uint32_t W = sizeof(T) * 8;                    // words
    uint32_t w[W];
    if (WIDE) {
#pragma unroll
        for (uint32_t i = 0; i < W; i += 8) ld_v8(p + 4 * i, w + i);
    } else if (sizeof(T) == 4) {
#pragma unroll
        for (uint32_t i = 0; i < W; ++i) w[i] = reinterpret_cast<const uint32_t*>(p)[i];
    } else {
#pragma unroll
        for (uint32_t i = 0; i < W; ++i) w[i] = reinterpret_cast<const uint16_t*>(p)[2 * i] | ((uint32_t)reinterpret_cast<const uint16_t*>(p)[2 * i + 1] << 16);
    }
#pragma unroll
    for (uint32_t i = 0; i < 32; ++i) {
        if constexpr (sizeof(T) == 4) v[i] = __uint_as_float(w[i]);
        else if constexpr (std::is_same<T, __nv_bfloat16>::value) v[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
        else { const float2 f = half_pair(w[i / 2]); v[i] = i & 1 ? f.y : f.x; }
    }
}
__device__ __forceinline__ void st_v8(void* p, const uint32_t v[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 :: "l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
template <typename T, bool WIDE>
__device__ __forceinline__ void store_block(uint8_t* p, const float v[32])
{
    constexpr uint32_t W = sizeof(T) * 8;
    uint32_t w[W];
#pragma unroll
    for (uint32_t i = 0; i < W; ++i) {
        if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(v[i]);
        else if constexpr (std::is_same<T, __nv_bfloat16>::value) { const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]); w[i] = *reinterpret_cast<const uint32_t*>(&h); }
        else { const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]); w[i] = *reinterpret_cast<const uint32_t*>(&h); }
    }
    if (WIDE) {
#pragma unroll
        for (uint32_t i = 0; i < W; i += 8) st_v8(p + 4 * i, w + i);
    } else if (sizeof(T) == 4) {
#pragma unroll
        for (uint32_t i = 0; i < W; ++i) reinterpret_cast<uint32_t*>(p)[i] = w[i];
    } else {
#pragma unroll
        for (uint32_t i = 0; i < W; ++i) {
            reinterpret_cast<uint16_t*>(p)[2 * i] = (uint16_t)w[i];
            reinterpret_cast<uint16_t*>(p)[2 * i + 1] = (uint16_t)(w[i] >> 16);
        }
    }
}

// ---- 32 elements of the cache ----
template <bool FP4>
struct Packed;
template <>
struct Packed<true> {
    uint32_t w[4];
    __device__ __forceinline__ uint32_t quantize(const float v[32])
    {
        float amax = 0.0f;
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const float a = fabsf(v[i]);
            odd |= !(a < __int_as_float(0x7F800000));
            amax = fmaxf(amax, a);
        }
        const uint32_t b = __float_as_uint(amax);
        const int e = (int)(b >> 23) - 127 - 2 + ((b & 0x7FFFFFu) > 0x400000u ? 1 : 0);      // 6 = 1.5 * 2^2
        const uint32_t s = odd ? 255u : b == 0 || e < -127 ? 0u : (uint32_t)(e + 127);
        const float inv = odd ? 0.0f : inverse_scale(s);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t r;
            asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
                "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
                "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
                "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
                : "=r"(r) : "f"(v[8 * i] * inv), "f"(v[8 * i + 1] * inv), "f"(v[8 * i + 2] * inv), "f"(v[8 * i + 3] * inv),
                            "f"(v[8 * i + 4] * inv), "f"(v[8 * i + 5] * inv), "f"(v[8 * i + 6] * inv), "f"(v[8 * i + 7] * inv));
            w[i] = odd ? 0u : r;
        }
        return s;
    }
    __device__ __forceinline__ void values(uint32_t s, float v[32]) const
    {
        const float f = e8m0_value(s);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t h[4];
            fp4_to_half(w[i], h);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 x = half_pair(h[j]);
                v[8 * i + 2 * j] = x.x * f;
                v[8 * i + 2 * j + 1] = x.y * f;
            }
        }
    }
};
template <>
struct Packed<false> {
    uint32_t w[8];
    __device__ __forceinline__ uint32_t quantize(const float v[32])
    {
        float amax = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) amax = fmaxf(amax, finite_abs(v[i]));
        const uint32_t s = scale_byte<false>(amax);
        const float inv = inverse_scale(s);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t r = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float x = v[4 * i + j];
                if (fabsf(x) == __int_as_float(0x7F800000)) x = __int_as_float(0x7FFFFFFF);          // there is no infinity
                r |= (uint32_t)__nv_cvt_float_to_fp8(x * inv, __NV_SATFINITE, __NV_E4M3) << (8 * j);
            }
            w[i] = r;
        }
        return s;
    }
    __device__ __forceinline__ void values(uint32_t s, float v[32]) const
    {
        const float f = e8m0_value(s);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t h[2];
            e4m3_to_half(w[i], h);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float2 x = half_pair(h[j]);
                v[4 * i + 2 * j] = x.x * f;
                v[4 * i + 2 * j + 1] = x.y * f;
            }
        }
    }
};

// A block's pieces in order: blocks of a token's head, rows, heads, keys and values.
struct Piece {
    uint32_t blk, row, head, side;
    __device__ __forceinline__ Piece(const CacheParams& P, uint32_t blocks, uint32_t i)
    {
        blk = i & (blocks - 1);
        i /= blocks;
        row = i & (P.rows_per_block - 1);
        i /= P.rows_per_block;
        side = i >= P.C.heads || P.sides == 2;
        head = i >= P.C.heads ? i - P.C.heads : i;
    }
};

template <typename T, bool FP4, uint32_t DIM, bool WIDE>
__global__ void __launch_bounds__(kCacheThreads) kv_append_kernel(const CacheParams P)
{
    __shared__ int places[kCacheMaxRows];
    constexpr uint32_t kBlocks = DIM / kKvBlock;
    grid_wait();
    grid_launch_dependents();
    const int row0 = (int)(blockIdx.x * P.rows_per_block);
    const uint32_t pieces = kBlocks * P.rows_per_block * P.C.heads * 2;
    const int first_row = P.B.first[0], end_row = min(P.B.first[P.B.n_seqs], (int)P.B.n_rows);        // the others are nobody's
    bool there = false;
    for (uint32_t i = threadIdx.x; i < pieces || !there; i += kCacheThreads) {
        const Piece c(P, kBlocks, i);
        const int row = row0 + (int)c.row;
        const bool mine = i < pieces && row >= first_row && row < end_row;
        float v[32];
        // the numbers do not wait for their place
        if (mine) load_block<T, WIDE>(P.t[c.side].d + (uint64_t)(row0 + c.row) * P.t[c.side].ld_row + c.head * P.t[c.side].ld_head + c.blk * kKvBlock * sizeof(T), v);
        if (!there) {
            find_places(P, row0, places);
            __syncthreads();
            there = true;
        }
        if (!mine || places[c.row] < 0) continue;
        Packed<FP4> q;
        const uint32_t s = q.quantize(v);
        const uint64_t at = block_at(P.C, places[c.row], c.head, kBlocks, c.blk);
        uint4* to = reinterpret_cast<uint4*>(P.C.elems[c.side] + at * sizeof q.w);
        to[0] = make_uint4(q.w[0], q.w[1], q.w[2], q.w[3]);
        if constexpr (!FP4) to[1] = make_uint4(q.w[4], q.w[5], q.w[6], q.w[7]);
        P.C.scales[c.side][at] = (uint8_t)s;
    }
}

template <typename T, bool FP4, uint32_t DIM, bool WIDE>
__global__ void __launch_bounds__(kCacheThreads) kv_read_kernel(const CacheParams P)
{
    __shared__ int places[kCacheMaxRows];
    constexpr uint32_t kBlocks = DIM / kKvBlock;
    grid_wait();
    grid_launch_dependents();
    const int row0 = (int)(blockIdx.x * P.rows_per_block);
    const uint32_t pieces = kBlocks * P.rows_per_block * P.C.heads * (P.sides == 3 ? 2 : 1);
    find_places(P, row0, places);
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < pieces; i += kCacheThreads) {
        const Piece c(P, kBlocks, i);
        const int place = places[c.row];
        if (place == -2) continue;
        float v[32];
        if (place < 0) {
#pragma unroll
            for (int k = 0; k < 32; ++k) v[k] = 0.0f;
        } else {
            Packed<FP4> q;
            const uint64_t at = block_at(P.C, place, c.head, kBlocks, c.blk);
            const uint8_t* from = P.C.elems[c.side] + at * sizeof q.w;
#pragma unroll
            for (uint32_t k = 0; k < sizeof q.w / 16; ++k) {
                const uint4 x = ld_stream_v4(from + 16 * k);
                q.w[4 * k] = x.x; q.w[4 * k + 1] = x.y; q.w[4 * k + 2] = x.z; q.w[4 * k + 3] = x.w;
            }
            q.values(P.C.scales[c.side][at], v);
        }
        store_block<T, WIDE>(P.t[c.side].d + (uint64_t)(row0 + c.row) * P.t[c.side].ld_row + c.head * P.t[c.side].ld_head + c.blk * kKvBlock * sizeof(T), v);
    }
}

template <typename T, bool FP4, uint32_t DIM, bool WIDE>
static cudaError_t launch_rows(const CacheParams& P, bool append, cudaStream_t st)
{
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute at[1] = {launch_early()};
    cfg.blockDim = dim3(kCacheThreads);
    cfg.gridDim = dim3((P.B.n_rows + P.rows_per_block - 1) / P.rows_per_block);
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return append ? cudaLaunchKernelEx(&cfg, kv_append_kernel<T, FP4, DIM, WIDE>, P) : cudaLaunchKernelEx(&cfg, kv_read_kernel<T, FP4, DIM, WIDE>, P);
}

static zc_status move_rows(bool append, const zc_kv_cache* cache, const zc_kv_batch* batch, zc_real type, const zc_kv_tensor* k, const zc_kv_tensor* v,
                           void* cuda_stream)
{
    const uint32_t width = real_bytes(type);
    if (!width) return ZC_E_UNSUPPORTED;
    if (const zc_status s = check_cache(cache)) return s;
    if (const zc_status s = check_batch(cache, batch)) return s;
    if (append ? !k || !v : !k && !v) return ZC_E_INVALID_ARG;
    if (batch->n_seqs == 0 || batch->n_rows == 0) return ZC_OK;
    bool wide = true;                                        // 32-byte pieces where every row and head begins on such a boundary
    for (const zc_kv_tensor* t : {k, v})
        if (t) {
            if (const zc_status s = check_tensor(t, width, batch->n_rows, cache->kv_heads, cache->head_dim)) return s;
            wide = wide && reinterpret_cast<uintptr_t>(t->d) % 32 == 0 && t->ld_row * width % 32 == 0 && t->ld_head * width % 32 == 0;
        }
    CacheParams P{};
    unsigned int* marks = kv_marks_word();
    if (!marks) return ZC_E_CUDA;
    P.C = device_cache(cache);
    P.B = device_batch(cache, batch, marks);
    P.t[0] = device_tensor(k, width);
    P.t[1] = device_tensor(v, width);
    P.sides = (k ? 1 : 0) | (v ? 2 : 0);
    P.rows_per_block = 1;
    while (P.rows_per_block < kCacheMaxRows && P.B.n_rows / P.rows_per_block > 2048) P.rows_per_block *= 2;
    cudaError_t e;
    auto with = [&](auto value) {
        using T = decltype(value);
        cudaStream_t st = (cudaStream_t)cuda_stream;
        auto dims = [&](auto fp4, auto w) {
            return cache->head_dim == 128 ? launch_rows<T, decltype(fp4)::value, 128, decltype(w)::value>(P, append, st)
                                          : launch_rows<T, decltype(fp4)::value, 64, decltype(w)::value>(P, append, st);
        };
        using Yes = std::true_type;
        using No = std::false_type;
        if (cache->format == ZC_FMT_FP4_E2M1) return wide ? dims(Yes(), Yes()) : dims(Yes(), No());
        return wide ? dims(No(), Yes()) : dims(No(), No());
    };
    if (type == ZC_REAL_F32) e = with(float());
    else if (type == ZC_REAL_BF16) e = with(__nv_bfloat16());
    else e = with(__half());
    return e == cudaSuccess ? ZC_OK : ZC_E_CUDA;
}

}  // namespace zc

using namespace zc;

extern "C" {

zc_status zc_kv_append(const zc_kv_cache* cache, const zc_kv_batch* batch, zc_real type, const zc_kv_tensor* k, const zc_kv_tensor* v, void* cuda_stream)
{
    return move_rows(true, cache, batch, type, k, v, cuda_stream);
}

zc_status zc_kv_read(const zc_kv_cache* cache, const zc_kv_batch* batch, zc_real type, const zc_kv_tensor* k, const zc_kv_tensor* v, void* cuda_stream)
{
    return move_rows(false, cache, batch, type, k, v, cuda_stream);
}

zc_status zc_kv_status(void* cuda_stream)
{
    static std::atomic<uint32_t> asked{0};
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(st, &capture) != cudaSuccess || capture != cudaStreamCaptureStatusNone) return ZC_E_CUDA;
    unsigned int *word = kv_marks_word(), marks = 0;
    if (!word) return ZC_E_CUDA;
    // every query has a place of its own for its answer, as long as no more than kKvAnswers threads ask at the same time
    const uint32_t at = asked.fetch_add(1, std::memory_order_relaxed) % kKvAnswers;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = cfg.blockDim = dim3(1);
    cfg.stream = st;
    if (cudaLaunchKernelEx(&cfg, kv_collect_kernel, word, at) != cudaSuccess) return ZC_E_CUDA;
    if (cudaMemcpyFromSymbolAsync(&marks, g_kv_answers, sizeof marks, at * sizeof marks, cudaMemcpyDeviceToHost, st) != cudaSuccess) return ZC_E_CUDA;
    if (cudaStreamSynchronize(st) != cudaSuccess) return ZC_E_CUDA;
    return marks & kKvGaveUp ? ZC_E_DEVICE_TIMEOUT : marks & kKvCorrupt ? ZC_E_CORRUPT : ZC_OK;
}

}  // extern "C"
