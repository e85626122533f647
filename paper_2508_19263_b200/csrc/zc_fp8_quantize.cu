// zc_fp8_quantize: FP32 / BF16 / FP16 matrices into FP8 elements and E8M0 scale bytes.
//
// For a block with largest finite magnitude amax = f * 2^E, 1 <= f < 2, and a format whose largest value is
// 1.75 * 2^Emax, the least e with amax <= 1.75 * 2^(Emax + e) is E - Emax, plus one when f > 1.75: the exponent and
// mantissa bits of amax give it exactly, without a logarithm or a division.  X * 2^-e is exact in FP32 wherever it is not
// far below the format's smallest value, so the one rounding is the conversion to FP8.
#include "zc_fp8.cuh"

namespace zc {

constexpr int kQuantThreads = 256;

struct QuantParams {
    const uint8_t* in;
    uint64_t ld_in;                              // bytes
    uint32_t rows, cols, col_blocks;
    uint8_t *q, *qs, *qt, *qts;                  // elements and scales of X and of its transposed form (null: not wanted)
    uint64_t ld_q, ld_qs, ld_qt, ld_qts;
};

template <typename T> struct RealOf;
template <> struct RealOf<float> { static __device__ __forceinline__ float get(float v) { return v; } };
template <> struct RealOf<__nv_bfloat16> { static __device__ __forceinline__ float get(__nv_bfloat16 v) { return __bfloat162float(v); } };
template <> struct RealOf<__half> { static __device__ __forceinline__ float get(__half v) { return __half2float(v); } };

// 16 consecutive elements, of which the first n exist (the others read as 0, which no maximum or sum notices).
template <typename T, bool WIDE>
__device__ __forceinline__ void load16(const uint8_t* p, uint32_t n, float v[16])
{
    if (WIDE && n >= 16) {
        if constexpr (sizeof(T) == 4) {
            uint32_t w[16];
            ld_v8(p, w);
            ld_v8(p + 32, w + 8);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(w[i]);
        } else {
            uint32_t w[8];
            ld_v8(p, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                T lo, hi;
                *reinterpret_cast<uint16_t*>(&lo) = (uint16_t)(w[i] & 0xFFFFu);
                *reinterpret_cast<uint16_t*>(&hi) = (uint16_t)(w[i] >> 16);
                v[2 * i] = RealOf<T>::get(lo);
                v[2 * i + 1] = RealOf<T>::get(hi);
            }
        }
        return;
    }
#pragma unroll
    for (uint32_t i = 0; i < 16; ++i) v[i] = i < n ? RealOf<T>::get(reinterpret_cast<const T*>(p)[i]) : 0.0f;
}

// Four elements times `inv` as FP8 bytes.  The conversion saturates infinities, so they are put right after it (rare).
template <bool E5M2>
__device__ __forceinline__ uint32_t to_fp8x4(const float v[4], float inv)
{
    const __nv_fp8_interpretation_t kind = E5M2 ? __NV_E5M2 : __NV_E4M3;
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[0] * inv, v[1] * inv), __NV_SATFINITE, kind);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[2] * inv, v[3] * inv), __NV_SATFINITE, kind);
    uint32_t r = lo | (hi << 16);
    if (isinf(v[0]) || isinf(v[1]) || isinf(v[2]) || isinf(v[3])) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (isinf(v[i])) r = (r & ~(0xFFu << (8 * i))) | (((E5M2 ? 0x7Cu : 0x7Fu) | (v[i] < 0 ? 0x80u : 0u)) << (8 * i));
    }
    return r;
}

__device__ __forceinline__ void store16(uint8_t* p, const uint32_t w[4], uint32_t n)
{
    if (n >= 16) {
        asm volatile("st.global.v4.b32 [%0], {%1,%2,%3,%4};" :: "l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
        return;
    }
#pragma unroll
    for (uint32_t i = 0; i < 16; ++i)
        if (i < n) p[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
}

// Blocks of 1 x 128, no transposed form: eight lanes a block, sixteen consecutive elements a lane.
template <typename T, bool E5M2, bool WIDE>
__global__ void __launch_bounds__(kQuantThreads)
quantize_rows_kernel(const __grid_constant__ QuantParams P)
{
    grid_launch_dependents();
    grid_wait();
    const uint32_t sub = threadIdx.x & 7;
    const uint32_t n_blocks = P.rows * P.col_blocks;
    const uint32_t block = (blockIdx.x * kQuantThreads + threadIdx.x) >> 3;
    // lanes behind the last block keep to the shuffles with nothing to load
    const uint32_t row = block / P.col_blocks, cb = block - row * P.col_blocks;
    const uint32_t col = cb * 128 + sub * 16;
    const uint32_t n = block < n_blocks && col < P.cols ? P.cols - col : 0;
    float v[16];
    load16<T, WIDE>(P.in + (uint64_t)row * P.ld_in + (uint64_t)col * sizeof(T), n, v);
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) amax = fmaxf(amax, finite_abs(v[i]));
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, d));
    const uint32_t s = scale_byte<E5M2>(amax);
    const float inv = inverse_scale(s);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = to_fp8x4<E5M2>(v + 4 * i, inv);
    if (n) store16(P.q + (uint64_t)row * P.ld_q + col, w, n);
    if (n && sub == 0) P.qs[(uint64_t)row * P.ld_qs + cb] = (uint8_t)s;
}

// A tile of 128 x 128 per thread block, held in registers (four rows of sixteen elements a thread) so that it is read
// once whatever comes of it: 128 x 128 blocks, and / or the transposed form, whose bytes change places in shared memory.
template <typename T, bool E5M2, bool WIDE, bool SQUARE, bool TRANS>
__global__ void __launch_bounds__(kQuantThreads)
quantize_tile_kernel(const __grid_constant__ QuantParams P)
{
    __shared__ __align__(16) uint32_t s_bytes[TRANS ? 128 * 32 : 1];     // [column][row / 4], turned by 4 words per 16 columns
    __shared__ float s_max[8][SQUARE ? 1 : 128];
    __shared__ uint32_t s_scale[SQUARE || !TRANS ? 1 : 128];
    grid_launch_dependents();
    grid_wait();
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rb = blockIdx.x / P.col_blocks, cb = blockIdx.x - rb * P.col_blocks;
    const uint32_t sub = tid & 7, rg = tid >> 3;
    const uint32_t row0 = rb * 128 + rg * 4, col0 = cb * 128 + sub * 16;
    const uint32_t n = col0 < P.cols ? P.cols - col0 : 0;
    float v[4][16];
#pragma unroll
    for (int p = 0; p < 4; ++p)
        load16<T, WIDE>(P.in + (uint64_t)(row0 + p) * P.ld_in + (uint64_t)col0 * sizeof(T), row0 + p < P.rows ? n : 0, v[p]);

    uint32_t row_scale[4];
    if constexpr (SQUARE) {
        float amax = 0.0f;
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int i = 0; i < 16; ++i) amax = fmaxf(amax, finite_abs(v[p][i]));
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, d));
        if (lane == 0) s_max[warp][0] = amax;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 8; ++k) amax = fmaxf(amax, s_max[k][0]);
        const uint32_t s = scale_byte<E5M2>(amax);
#pragma unroll
        for (int p = 0; p < 4; ++p) row_scale[p] = s;
        if (tid == 0) {
            if (P.q) P.qs[(uint64_t)rb * P.ld_qs + cb] = (uint8_t)s;
            if (TRANS) P.qts[(uint64_t)cb * P.ld_qts + rb] = (uint8_t)s;
        }
    } else {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            float amax = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) amax = fmaxf(amax, finite_abs(v[p][i]));
#pragma unroll
            for (int d = 1; d < 8; d <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, d));
            row_scale[p] = scale_byte<E5M2>(amax);
            if (P.q && sub == 0 && row0 + p < P.rows) P.qs[(uint64_t)(row0 + p) * P.ld_qs + cb] = (uint8_t)row_scale[p];
        }
        // the columns' maxima: over a thread's four rows, the warp's sixteen, the block's 128
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float m = fmaxf(fmaxf(finite_abs(v[0][i]), finite_abs(v[1][i])), fmaxf(finite_abs(v[2][i]), finite_abs(v[3][i])));
            m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 8));
            m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
            if (lane < 8) s_max[warp][sub * 16 + i] = m;
        }
        __syncthreads();
        if (tid < 128) {
            float m = 0.0f;
#pragma unroll
            for (int k = 0; k < 8; ++k) m = fmaxf(m, s_max[k][tid]);
            const uint32_t s = scale_byte<E5M2>(m);
            s_scale[tid] = s;
            if (cb * 128 + tid < P.cols) P.qts[(uint64_t)(cb * 128 + tid) * P.ld_qts + rb] = (uint8_t)s;
        }
        __syncthreads();
    }
    if (P.q) {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            if (row0 + p >= P.rows || n == 0) continue;
            const float inv = inverse_scale(row_scale[p]);
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = to_fp8x4<E5M2>(v[p] + 4 * i, inv);
            store16(P.q + (uint64_t)(row0 + p) * P.ld_q + col0, w, n);
        }
    }
    if constexpr (TRANS) {
        // four rows of a column make a word; words of a column are turned so that a warp's 32 stores fall into 32 banks
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float inv = inverse_scale(SQUARE ? row_scale[0] : s_scale[sub * 16 + i]);
            const float c[4] = {v[0][i], v[1][i], v[2][i], v[3][i]};
            s_bytes[(sub * 16 + i) * 32 + ((rg + 4 * sub) & 31)] = to_fp8x4<E5M2>(c, inv);
        }
        __syncthreads();
        const uint32_t r0 = rb * 128 + sub * 16;
        const uint32_t nr = r0 < P.rows ? P.rows - r0 : 0;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const uint32_t c = p * 32 + rg;
            const uint4 x = *reinterpret_cast<const uint4*>(&s_bytes[c * 32 + ((4 * sub + 4 * (c >> 4)) & 31)]);
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
            if (cb * 128 + c < P.cols && nr) store16(P.qt + (uint64_t)(cb * 128 + c) * P.ld_qt + r0, w, nr);
        }
    }
}

template <typename T, bool E5M2, bool WIDE>
static cudaError_t launch_quantize(const QuantParams& P, bool square, uint32_t n_blocks, uint32_t n_tiles, cudaStream_t st)
{
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute at[1] = {launch_early()};
    cfg.blockDim = dim3(kQuantThreads);
    cfg.gridDim = dim3(square || P.qt ? n_tiles : (n_blocks + kQuantThreads / 8 - 1) / (kQuantThreads / 8));
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (square && P.qt) return cudaLaunchKernelEx(&cfg, quantize_tile_kernel<T, E5M2, WIDE, true, true>, P);
    if (square) return cudaLaunchKernelEx(&cfg, quantize_tile_kernel<T, E5M2, WIDE, true, false>, P);
    if (P.qt) return cudaLaunchKernelEx(&cfg, quantize_tile_kernel<T, E5M2, WIDE, false, true>, P);
    return cudaLaunchKernelEx(&cfg, quantize_rows_kernel<T, E5M2, WIDE>, P);
}

}  // namespace zc

using namespace zc;

extern "C" zc_status zc_fp8_quantize(zc_real in_type, const void* d_in, uint64_t ld_in, const zc_fp8_matrix* q,
                                     const zc_fp8_matrix* qt, void* cuda_stream)
{
    if (!q && !qt) return ZC_E_INVALID_ARG;
    const uint32_t width = real_bytes(in_type);
    if (!width) return ZC_E_UNSUPPORTED;
    for (const zc_fp8_matrix* m : {q, qt})
        if (m)
            if (const zc_status s = check_matrix(m)) return s;
    const uint64_t rows = q ? q->rows : qt->cols, cols = q ? q->cols : qt->rows;
    if (q && qt && (qt->rows != cols || qt->cols != rows || q->format != qt->format || q->block_rows != qt->block_rows)) return ZC_E_INVALID_ARG;
    if (rows == 0 || cols == 0) return ZC_OK;
    if (!d_in || reinterpret_cast<uintptr_t>(d_in) % width || ld_in < cols || ld_in >= (1ull << 39)) return ZC_E_INVALID_ARG;
    const uint64_t n_blocks = rows * ceil_div(cols, 128), n_tiles = ceil_div(rows, 128) * ceil_div(cols, 128);
    if (n_blocks >= (1ull << 32) - 64 || n_tiles >= (1ull << 31)) return ZC_E_TOO_LARGE;
    QuantParams P{};
    P.in = (const uint8_t*)d_in;
    P.ld_in = ld_in * width;
    P.rows = (uint32_t)rows;
    P.cols = (uint32_t)cols;
    P.col_blocks = (uint32_t)ceil_div(cols, 128);
    if (q) { P.q = (uint8_t*)q->d_elems; P.qs = (uint8_t*)q->d_scales; P.ld_q = q->ld_elems; P.ld_qs = q->ld_scales; }
    if (qt) { P.qt = (uint8_t*)qt->d_elems; P.qts = (uint8_t*)qt->d_scales; P.ld_qt = qt->ld_elems; P.ld_qts = qt->ld_scales; }
    const zc_fp8_matrix* any = q ? q : qt;
    const bool square = any->block_rows == 128, e5m2 = any->format == ZC_FMT_FP8_E5M2;
    // 32-byte loads where every row begins on a 32-byte boundary
    const bool wide = reinterpret_cast<uintptr_t>(d_in) % 32 == 0 && P.ld_in % 32 == 0;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e;
    auto run = [&](auto value) {
        using T = decltype(value);
        const uint32_t nb = (uint32_t)n_blocks, nt = (uint32_t)n_tiles;
        return e5m2 ? (wide ? launch_quantize<T, true, true>(P, square, nb, nt, st) : launch_quantize<T, true, false>(P, square, nb, nt, st))
                    : (wide ? launch_quantize<T, false, true>(P, square, nb, nt, st) : launch_quantize<T, false, false>(P, square, nb, nt, st));
    };
    if (in_type == ZC_REAL_F32) e = run(float());
    else if (in_type == ZC_REAL_BF16) e = run(__nv_bfloat16());
    else e = run(__half());
    return e == cudaSuccess ? ZC_OK : ZC_E_CUDA;
}
