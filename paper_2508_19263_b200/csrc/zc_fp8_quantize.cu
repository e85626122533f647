// zc_fp8_quantize: FP32 / BF16 / FP16 matrices into FP8 elements and E8M0 scale bytes.
//
// For a block with largest finite magnitude amax = f * 2^E, 1 <= f < 2, and a format whose largest value is
// 1.75 * 2^Emax, the least e with amax <= 1.75 * 2^(Emax + e) is E - Emax, plus one when f > 1.75: the exponent and
// mantissa bits of amax give it exactly, without a logarithm or a division.  X * 2^-e is exact in FP32 wherever it is not
// far below the format's smallest value, so the one rounding is the conversion to FP8.
#include <type_traits>

#include "zc_fp8.cuh"

namespace zc {

constexpr int kQuantThreads = 256;

struct QuantParams {
    const uint8_t *in, *in_end;                  // first byte, and the one behind the last
    uint64_t ld_in;                              // bytes
    uint32_t rows, cols, col_blocks;
    uint8_t *q, *qs, *qt, *qts;                  // elements and scales of X and of its transposed form (null: not wanted)
    uint64_t ld_q, ld_qs, ld_qt, ld_qts;
};

// Sixteen consecutive elements as they were loaded: pairs of 16-bit ones to a word, or a word each.
template <typename T>
struct Raw {
    static constexpr int kWords = sizeof(T) == 4 ? 16 : 8;
    static constexpr uint32_t kInfinity = sizeof(T) == 4 ? 0x7F800000u : std::is_same<T, __half>::value ? 0x7C00u : 0x7F80u;
    uint32_t w[kWords];

    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else if constexpr (std::is_same<T, __nv_bfloat16>::value) return __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
        else return __half2float(__ushort_as_half((uint16_t)(w[i >> 1] >> (16 * (i & 1)))));
    }
    // Magnitudes order like their bits: maxima are taken on these, of two 16-bit elements at a time.
    static __device__ __forceinline__ uint32_t magnitude(uint32_t x) { return sizeof(T) == 4 ? x & 0x7FFFFFFFu : x & 0x7FFF7FFFu; }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return sizeof(T) == 4 ? max(a, b) : __vmaxu2(a, b); }
    // whether one of a word's magnitudes is an infinity or NaN
    static __device__ __forceinline__ bool endless(uint32_t m)
    {
        return sizeof(T) == 4 ? m >= kInfinity : (m & 0xFFFFu) >= kInfinity || (m >> 16) >= kInfinity;
    }
    // a word's magnitudes, 0 in the place of infinities and NaN
    static __device__ __forceinline__ uint32_t finite(uint32_t x)
    {
        const uint32_t m = magnitude(x);
        if (sizeof(T) == 4) return m >= kInfinity ? 0u : m;
        return ((m & 0xFFFFu) >= kInfinity ? 0u : m & 0xFFFFu) | ((m >> 16) >= kInfinity ? 0u : m & 0xFFFF0000u);
    }
    // a magnitude (of the lower element of a word, where it holds two) as FP32 bits
    static __device__ __forceinline__ uint32_t as_f32(uint32_t m)
    {
        if constexpr (sizeof(T) == 4) return m;
        else if constexpr (std::is_same<T, __nv_bfloat16>::value) return m << 16;
        else return __float_as_uint(__half2float(__ushort_as_half((uint16_t)m)));
    }
    // the larger of a word's magnitudes
    static __device__ __forceinline__ uint32_t one(uint32_t m) { return sizeof(T) == 4 ? m : max(m & 0xFFFFu, m >> 16); }
};

// 16 consecutive elements, of which the first n exist (the others read as 0, which no maximum notices).  WIDE: 32-byte
// loads are aligned.  Otherwise the aligned 16-byte pieces that hold the elements are loaded and shifted into place, where they lie
// inside the matrix (777 x 11009 in FP16: 12.3 us with loads of single elements, 6.5 so).
template <typename T, bool WIDE>
__device__ __forceinline__ Raw<T> load16(const QuantParams& P, const uint8_t* p, uint32_t n)
{
    Raw<T> r;
    constexpr int W = Raw<T>::kWords;
    const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15);
    if (n >= 16 && WIDE) {
        ld_v8(p, r.w);
        if constexpr (W == 16) ld_v8(p + 32, r.w + 8);
    } else if (n >= 16 && p - off >= P.in && p - off + 4 * W + 16 <= P.in_end) {
        uint32_t u[W + 4];
#pragma unroll
        for (int i = 0; i < W / 4 + 1; ++i) {
            const uint4 v = ld_stream_v4(p - off + 16 * i);
            u[4 * i] = v.x; u[4 * i + 1] = v.y; u[4 * i + 2] = v.z; u[4 * i + 3] = v.w;
        }
        if (off & 8)
#pragma unroll
            for (int i = 0; i < W + 2; ++i) u[i] = u[i + 2];
        if (off & 4)
#pragma unroll
            for (int i = 0; i < W + 1; ++i) u[i] = u[i + 1];
#pragma unroll
        for (int i = 0; i < W; ++i) r.w[i] = sizeof(T) == 4 ? u[i] : __funnelshift_r(u[i], u[i + 1], 8 * (off & 3));
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if constexpr (sizeof(T) == 4) {
                r.w[i] = (uint32_t)i < n ? reinterpret_cast<const uint32_t*>(p)[i] : 0u;
            } else {
                const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
                r.w[i] = ((uint32_t)(2 * i) < n ? q[2 * i] : 0u) | ((uint32_t)(2 * i + 1) < n ? (uint32_t)q[2 * i + 1] << 16 : 0u);
            }
        }
    }
    return r;
}

// The largest finite magnitude of 16 elements, as one() gives it; `odd`: there are infinities or NaN among them.
template <typename T>
__device__ __forceinline__ uint32_t largest(const Raw<T>& r, bool& odd)
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < Raw<T>::kWords; ++i) m = Raw<T>::larger(m, Raw<T>::magnitude(r.w[i]));
    odd = Raw<T>::endless(m);
    if (odd) {
        m = 0;
#pragma unroll
        for (int i = 0; i < Raw<T>::kWords; ++i) m = Raw<T>::larger(m, Raw<T>::finite(r.w[i]));
    }
    return Raw<T>::one(m);
}
template <typename T, bool E5M2>
__device__ __forceinline__ uint32_t scale_of(uint32_t m) { return scale_byte<E5M2>(__uint_as_float(Raw<T>::as_f32(m))); }

// Four elements times `inv` as FP8 bytes.  The conversion saturates infinities, so they are put right after it (`odd`, rare).
template <bool E5M2>
__device__ __forceinline__ uint32_t to_fp8x4(const float v[4], float inv, bool odd)
{
    const __nv_fp8_interpretation_t kind = E5M2 ? __NV_E5M2 : __NV_E4M3;
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[0] * inv, v[1] * inv), __NV_SATFINITE, kind);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[2] * inv, v[3] * inv), __NV_SATFINITE, kind);
    uint32_t r = lo | (hi << 16);
    if (odd) {
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

// Blocks of 1 x 128, no transposed form: eight lanes a block, sixteen consecutive elements a lane.  Bound by memory.
template <typename T, bool E5M2, bool WIDE>
__global__ void __launch_bounds__(kQuantThreads)
quantize_rows_kernel(const __grid_constant__ QuantParams P)
{
    const uint32_t sub = threadIdx.x & 7;
    const uint32_t n_blocks = P.rows * P.col_blocks;
    const uint32_t block = blockIdx.x * (kQuantThreads / 8) + (threadIdx.x >> 3);    // the threads' numbers would pass 32 bits
    // lanes behind the last block keep to the shuffles with nothing to load
    const uint32_t row = block / P.col_blocks, cb = block - row * P.col_blocks;
    const uint32_t col = cb * 128 + sub * 16;
    const uint32_t n = block < n_blocks && col < P.cols ? P.cols - col : 0;
    grid_wait();
    grid_launch_dependents();
    const Raw<T> r = load16<T, WIDE>(P, P.in + (uint64_t)row * P.ld_in + (uint64_t)col * sizeof(T), n);
    bool odd;
    uint32_t m = largest(r, odd);
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
    const uint32_t s = scale_of<T, E5M2>(m);
    const float inv = inverse_scale(s);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float v[4] = {r.get(4 * i), r.get(4 * i + 1), r.get(4 * i + 2), r.get(4 * i + 3)};
        w[i] = to_fp8x4<E5M2>(v, inv, odd);
    }
    if (n) store16(P.q + (uint64_t)row * P.ld_q + col, w, n);
    if (n && sub == 0) P.qs[(uint64_t)row * P.ld_qs + cb] = (uint8_t)s;
}

// A tile of 128 x 128 per thread block, held in registers as it was loaded (four rows of sixteen elements a thread), so that it is
// read once whatever comes of it: 128 x 128 blocks, and / or the transposed form, whose bytes change places in shared memory.
template <typename T, bool E5M2, bool WIDE, bool SQUARE, bool TRANS>
__global__ void __launch_bounds__(kQuantThreads, sizeof(T) == 4 ? 2 : 3)
quantize_tile_kernel(const __grid_constant__ QuantParams P)
{
    using R = Raw<T>;
    constexpr int W = R::kWords;
    __shared__ __align__(16) uint32_t s_bytes[TRANS ? 128 * 32 : 1];     // [column][row / 4], turned by 4 words per 16 columns
    __shared__ uint32_t s_max[8][SQUARE ? 1 : 8 * W];
    __shared__ uint32_t s_scale[SQUARE || !TRANS ? 1 : 128];
    grid_wait();
    grid_launch_dependents();
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rb = blockIdx.x / P.col_blocks, cb = blockIdx.x - rb * P.col_blocks;
    const uint32_t sub = tid & 7, rg = tid >> 3;
    const uint32_t row0 = rb * 128 + rg * 4, col0 = cb * 128 + sub * 16;
    const uint32_t n = col0 < P.cols ? P.cols - col0 : 0;
    R r[4];
#pragma unroll
    for (int p = 0; p < 4; ++p)
        r[p] = load16<T, WIDE>(P, P.in + (uint64_t)(row0 + p) * P.ld_in + (uint64_t)col0 * sizeof(T), row0 + p < P.rows ? n : 0);

    bool odd = false;
    uint32_t row_scale[4], m[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        bool o;
        m[p] = largest(r[p], o);
        odd = odd || o;
    }
    if constexpr (SQUARE) {
        const uint32_t all = __reduce_max_sync(0xFFFFFFFFu, max(max(m[0], m[1]), max(m[2], m[3])));
        if (lane == 0) s_max[warp][0] = all;
        __syncthreads();
        uint32_t most = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) most = max(most, s_max[k][0]);
        const uint32_t s = scale_of<T, E5M2>(most);
#pragma unroll
        for (int p = 0; p < 4; ++p) row_scale[p] = s;
        if (tid == 0) {
            if (P.q) P.qs[(uint64_t)rb * P.ld_qs + cb] = (uint8_t)s;
            if (TRANS) P.qts[(uint64_t)cb * P.ld_qts + rb] = (uint8_t)s;
        }
    } else {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
#pragma unroll
            for (int d = 1; d < 8; d <<= 1) m[p] = max(m[p], __shfl_xor_sync(0xFFFFFFFFu, m[p], d));
            row_scale[p] = scale_of<T, E5M2>(m[p]);
            if (P.q && sub == 0 && row0 + p < P.rows) P.qs[(uint64_t)(row0 + p) * P.ld_qs + cb] = (uint8_t)row_scale[p];
        }
        // the columns' maxima, two columns to a word of 16-bit elements: over a thread's four rows, the warp's sixteen, the block's 128
#pragma unroll
        for (int i = 0; i < W; ++i) {
            uint32_t c;
            if (odd) c = R::larger(R::larger(R::finite(r[0].w[i]), R::finite(r[1].w[i])), R::larger(R::finite(r[2].w[i]), R::finite(r[3].w[i])));
            else c = R::larger(R::larger(R::magnitude(r[0].w[i]), R::magnitude(r[1].w[i])), R::larger(R::magnitude(r[2].w[i]), R::magnitude(r[3].w[i])));
            c = R::larger(c, __shfl_xor_sync(0xFFFFFFFFu, c, 8));
            c = R::larger(c, __shfl_xor_sync(0xFFFFFFFFu, c, 16));
            if (lane < 8) s_max[warp][sub * W + i] = c;
        }
        __syncthreads();
        if (tid < 8 * W) {
            uint32_t c = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) c = R::larger(c, s_max[k][tid]);
#pragma unroll
            for (int h = 0; h < 16 / W; ++h) {
                const uint32_t at = tid * (16 / W) + h, s = scale_of<T, E5M2>(W == 16 ? c : h ? c >> 16 : c & 0xFFFFu);
                s_scale[at] = s;
                if (cb * 128 + at < P.cols) P.qts[(uint64_t)(cb * 128 + at) * P.ld_qts + rb] = (uint8_t)s;
            }
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
            for (int i = 0; i < 4; ++i) {
                const float v[4] = {r[p].get(4 * i), r[p].get(4 * i + 1), r[p].get(4 * i + 2), r[p].get(4 * i + 3)};
                w[i] = to_fp8x4<E5M2>(v, inv, odd);
            }
            store16(P.q + (uint64_t)(row0 + p) * P.ld_q + col0, w, n);
        }
    }
    if constexpr (TRANS) {
        // four rows of a column make a word; words of a column are turned so that a warp's 32 stores fall into 32 banks
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float inv = inverse_scale(SQUARE ? row_scale[0] : s_scale[sub * 16 + i]);
            const float c[4] = {r[0].get(i), r[1].get(i), r[2].get(i), r[3].get(i)};
            s_bytes[(sub * 16 + i) * 32 + ((rg + 4 * sub) & 31)] = to_fp8x4<E5M2>(c, inv, odd);
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
    P.in_end = P.in + (rows - 1) * P.ld_in + cols * width;
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
