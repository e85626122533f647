// What the attention kernels share: parameters, sequences cut into items, columns of an item, results.
#pragma once
#include "zc_fp8_tensor.cuh"
#include "zc_kv.cuh"

namespace zc {

struct AttentionParams {
    KvCache C;
    KvBatch B;
    KvTensor q, out;
    float* lse;
    uint8_t* workspace;
    uint32_t q_heads, group;
    float scale_mantissa;               // scale * log2(e), since exponentials are powers of two: +-1 .. 2, times 2^scale_exponent
    int scale_exponent;
    uint32_t causal, window;
    uint32_t half_type;                 // queries and results in FP16, else BF16
    uint32_t q_wide, out_wide;          // four neighbours begin on 8 bytes
    uint32_t most_rows;                 // sequences of up to so many rows are for the kernel of few rows, the others for that of many; all ones: all are
    uint32_t spin_limit, skip_copy, skip_math;
};

// An item's columns, as whoever joins its parts needs them.
struct ItemColumns {
    int row0;
    uint32_t head, first, count;             // columns first .. first + count - 1
};
// What a block leaves of the item that begins in it and goes on in the next ones.
struct BlockEnd {
    unsigned long long to, total;
    ItemColumns columns;
    uint32_t there, pad[3];
};

__device__ __forceinline__ float exp2_fast(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// Of a sum of weights, the largest of which is about 2^15, over 2^unit.
__device__ __forceinline__ float lse_of(float unit, float weight) { return weight == 0.0f ? -INFINITY : (unit + 15.0f + log2f(weight * (1.0f / 32768.0f))) * 0.69314718f; }
// whether one of four E4M3 bytes is NaN
__device__ __forceinline__ bool nan_bytes(uint32_t w)
{
    const uint32_t x = ~w & 0x7F7F7F7Fu;                                   // a byte of 0 where it is
    return ((x - 0x01010101u) & ~x & 0x80808080u) != 0;
}

__device__ __forceinline__ uint32_t lds16(uint32_t a) { uint16_t v; asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(a) : "memory"); return v; }
__device__ __forceinline__ void lds64(uint32_t a, uint32_t& x, uint32_t& y) { asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(x), "=r"(y) : "r"(a) : "memory"); }
__device__ __forceinline__ void lds_f2(uint32_t a, float v[2]) { asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(v[0]), "=f"(v[1]) : "r"(a) : "memory"); }
__device__ __forceinline__ void lds_f4(uint32_t a, float v[4]) { asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(a) : "memory"); }
__device__ __forceinline__ void sts16(uint32_t a, uint32_t v) { asm volatile("st.shared.u16 [%0], %1;" :: "r"(a), "h"((uint16_t)v) : "memory"); }
__device__ __forceinline__ void sts64(uint32_t a, uint32_t x, uint32_t y) { asm volatile("st.shared.v2.b32 [%0], {%1,%2};" :: "r"(a), "r"(x), "r"(y) : "memory"); }
__device__ __forceinline__ void sts_f1(uint32_t a, float v) { asm volatile("st.shared.f32 [%0], %1;" :: "r"(a), "f"(v) : "memory"); }
__device__ __forceinline__ void sts_f2(uint32_t a, const float* v) { asm volatile("st.shared.v2.f32 [%0], {%1,%2};" :: "r"(a), "f"(v[0]), "f"(v[1]) : "memory"); }
__device__ __forceinline__ void sts_f4(uint32_t a, const float* v) { asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};" :: "r"(a), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]) : "memory"); }
// Contiguous bytes to shared memory: 16-byte aligned on both sides, a multiple of 16.
__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" :: "r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// Waits of these kernels: bounded, and over for every role when one has given up, which is looked for at every kPolls-th poll only: warps that poll take the
// issue slots of those that work, so a poll is as few instructions as it can be (with a look at every poll, half of a many-row step's instructions were polls).
constexpr uint32_t kPolls = 32;
__device__ __forceinline__ bool bar_poll(uint32_t bar, uint32_t parity, uint32_t polls)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p, q;\n\t.reg .u32 n;\n\tmov.u32 n, %3;\n"
                 "AGAIN_%=:\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t@p bra OVER_%=;\n\t"
                 "sub.u32 n, n, 1;\n\tsetp.ne.u32 q, n, 0;\n\t@q bra AGAIN_%=;\n"
                 "OVER_%=:\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity), "r"(polls) : "memory");
    return ok != 0;
}
struct KvWaiter {
    uint32_t limit, failed;                              // failed: shared address of the block's mark
    __device__ __forceinline__ void give_up() const { asm volatile("st.volatile.shared.u32 [%0], 1;" :: "r"(failed) : "memory"); }
    // all lanes of a converged warp
    __device__ __forceinline__ bool warp(uint32_t bar, uint32_t parity) const
    {
        uint32_t left = limit;
        while (true) {
            const uint32_t some = min(left, kPolls - 1) + 1;
            if (__all_sync(0xFFFFFFFFu, bar_poll(bar, parity, some))) return true;
            uint32_t over;
            asm volatile("ld.volatile.shared.u32 %0, [%1];" : "=r"(over) : "r"(failed) : "memory");
            if (__any_sync(0xFFFFFFFFu, over != 0)) return false;
            if (left < some) { give_up(); return false; }
            left -= some;
        }
    }
};

// The rows of a sequence and the tokens that any of them sees.
struct SeqRows {
    int n, row0, len, from, to;
    __device__ __forceinline__ void load(const AttentionParams& P, uint32_t b)
    {
        const int first = P.B.first[b], last = P.B.first[b + 1];
        len = kv_len(P.B, b);
        row0 = first;
        n = 0;
        if (first >= 0 && last >= first && (uint32_t)last <= P.B.n_rows) n = last - first;
        else atomicOr(P.B.marks, kKvCorrupt);
        to = len;
        from = P.window ? (int)max(0ll, (long long)len - n + 1 - P.window) : 0;
    }
    // the tokens that a row sees
    __device__ __forceinline__ void limits(const AttentionParams& P, int j, int& lo, int& hi) const
    {
        const int pos = len - n + j;
        hi = P.causal ? pos + 1 : len;
        lo = P.window ? (int)max(0ll, (long long)pos + 1 - P.window) : 0;
    }
};

// A sequence as items of COLS columns and a head, `steps` steps each; a lane has one of 32 neighbouring sequences.
struct SeqSpan {
    SeqRows r;
    uint32_t tiles, steps;
    __device__ __forceinline__ unsigned long long cost(uint32_t heads) const { return (unsigned long long)tiles * heads * steps; }
};
template <uint32_t COLS, uint32_t STEP>
__device__ __forceinline__ SeqSpan stream_span(const AttentionParams& P, uint32_t b)
{
    SeqSpan s{};
    s.steps = 1;
    if (b < P.B.n_seqs) {
        s.r.load(P, b);
        if ((uint32_t)s.r.n <= P.most_rows) s.tiles = (uint32_t)(((unsigned long long)s.r.n * P.group + COLS - 1) / COLS);
        const uint32_t first = (uint32_t)s.r.from / STEP, last = ((uint32_t)s.r.to + STEP - 1) / STEP;
        s.steps = last > first ? last - first : 1;         // at least one, that rows which see nothing get their zeros
    }
    return s;
}

// Where a warp is.  All lanes have the same.
template <uint32_t COLS, uint32_t STEP>
struct Cursor : SeqRows {
    uint32_t b, item, head, tile, step, steps, tiles;
    __device__ __forceinline__ void take(const SeqSpan& s)
    {
        const uint32_t k = b & 31;
        n = __shfl_sync(0xFFFFFFFFu, s.r.n, k);
        row0 = __shfl_sync(0xFFFFFFFFu, s.r.row0, k);
        len = __shfl_sync(0xFFFFFFFFu, s.r.len, k);
        from = __shfl_sync(0xFFFFFFFFu, s.r.from, k);
        to = __shfl_sync(0xFFFFFFFFu, s.r.to, k);
        steps = __shfl_sync(0xFFFFFFFFu, s.steps, k);
        tiles = __shfl_sync(0xFFFFFFFFu, s.tiles, k);
    }
    __device__ __forceinline__ void place()
    {
        head = tiles > 1 ? item / tiles : item;
        tile = tiles > 1 ? item % tiles : 0;
    }
    __device__ __forceinline__ void set(const SeqSpan& s, uint32_t b_, uint32_t item_, uint32_t step_)
    {
        b = b_;
        item = item_;
        step = step_;
        take(s);
        place();
    }
    __device__ __forceinline__ uint32_t token() const { return ((uint32_t)from / STEP + step) * STEP; }
    __device__ __forceinline__ bool last() const { return step + 1 == steps; }
    __device__ __forceinline__ void next(const AttentionParams& P, SeqSpan& s)
    {
        if (++step < steps) return;
        step = 0;
        if (++item < tiles * P.C.heads) { place(); return; }
        item = 0;
        while (true) {
            if (++b >= P.B.n_seqs) return;
            if ((b & 31) == 0) s = stream_span<COLS, STEP>(P, b + (threadIdx.x & 31));
            if (__shfl_sync(0xFFFFFFFFu, s.tiles, b & 31)) break;
        }
        take(s);
        place();
    }
    __device__ __forceinline__ ItemColumns columns(const AttentionParams& P) const
    {
        return ItemColumns{row0, head, tile * COLS, min(COLS, (uint32_t)n * P.group - tile * COLS)};
    }
    __device__ __forceinline__ bool has(const AttentionParams& P, uint32_t col) const { return col < (uint32_t)n * P.group; }
    __device__ __forceinline__ void column_limits(const AttentionParams& P, uint32_t col, int& lo, int& hi) const
    {
        lo = 0;
        hi = 0x7FFFFFFF;
        if (has(P, col)) limits(P, (int)(col / P.group), lo, hi);
    }
    __device__ __forceinline__ const uint8_t* query(const AttentionParams& P, uint32_t col) const
    {
        return P.q.d + (uint64_t)(row0 + col / P.group) * P.q.ld_row + (uint64_t)(head * P.group + col % P.group) * P.q.ld_head;
    }
    __device__ __forceinline__ uint8_t* out(const AttentionParams& P, uint32_t col) const
    {
        return P.out.d + (uint64_t)(row0 + col / P.group) * P.out.ld_row + (uint64_t)(head * P.group + col % P.group) * P.out.ld_head;
    }
    __device__ __forceinline__ uint64_t lse(const AttentionParams& P, uint32_t col) const
    {
        return (uint64_t)(row0 + col / P.group) * P.q_heads + head * P.group + col % P.group;
    }
};

// N (2 or 4) neighbours of a result, from d on.
template <uint32_t N>
__device__ __forceinline__ void store_out(const AttentionParams& P, uint8_t* out, uint32_t d, const float* v)
{
    uint32_t w[N / 2];
#pragma unroll
    for (uint32_t k = 0; k < N / 2; ++k) {
        if (P.half_type) { const __half2 h = __floats2half2_rn(v[2 * k], v[2 * k + 1]); w[k] = *reinterpret_cast<const uint32_t*>(&h); }
        else { const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]); w[k] = *reinterpret_cast<const uint32_t*>(&h); }
    }
    out += 2 * d;
    if (P.out_wide) {
        if (N == 4) *reinterpret_cast<uint2*>(out) = make_uint2(w[0], w[N / 2 - 1]);
        else *reinterpret_cast<uint32_t*>(out) = w[0];
    } else {
#pragma unroll
        for (uint32_t k = 0; k < N; ++k) reinterpret_cast<uint16_t*>(out)[k] = (uint16_t)(w[k / 2] >> (16 * (k & 1)));
    }
}
// What divides sums by their weights; 0 where nothing was seen.  Off by 2^-22: results are rounded to 2^-9 or 2^-12.  (A correctly rounded one takes 0.5 us of a short call's 16.)
__device__ __forceinline__ float inverse_weight(float weight) { return weight == 0.0f ? 0.0f : __fdividef(1.0f, weight); }
// A joined column: a lane has N neighbours from d on.
template <uint32_t N>
__device__ __forceinline__ void finish_column(const AttentionParams& P, const ItemColumns& c, uint32_t in_tile, uint32_t d, const float* v, float top, float weight)
{
    const uint32_t col = c.first + in_tile, head = c.head * P.group + col % P.group;
    const uint64_t row = (uint64_t)c.row0 + col / P.group;
    store_out<N>(P, P.out.d + row * P.out.ld_row + head * P.out.ld_head, d, v);
    if (P.lse && d == 0) P.lse[row * P.q_heads + head] = lse_of(top, weight);
}

// Two neighbours of a query as FP32.
__device__ __forceinline__ float2 query_pair(const AttentionParams& P, uint32_t w)
{
    return P.half_type ? half_pair(w) : make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ uint2 query_four(const AttentionParams& P, const uint8_t* p)
{
    if (P.q_wide) return *reinterpret_cast<const uint2*>(p);
    const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
    return make_uint2(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16);
}
// The power of two that brings `most` to 2^14 .. 2^15, as far as FP32 goes; 1 where there is none.
__device__ __forceinline__ int query_lift(float most)
{
    const uint32_t e = __float_as_uint(most) >> 23;
    return e == 255 || most == 0.0f ? 0 : min(14 - ((int)e - 127), 126);
}
__device__ __forceinline__ float power_of_two(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }      // -126 .. 127
// What makes a logit (times log2(e)) of a product that is over 2^-e, as far as FP32's normal numbers go.  Above 0, that the largest product is the largest logit
// and -infinity stays: the scale's sign is with the queries.  One power of two for scale, queries and keys together: each for itself may be beyond FP32 where the logit is not.
// Without the scale's mantissa (its bits are scale_mantissa_bits) for who has that with the keys' scales.
__device__ __forceinline__ float logit_power(const AttentionParams& P, int e) { return __uint_as_float((uint32_t)min(max(P.scale_exponent + e + 127, 1), 254) << 23); }
__device__ __forceinline__ uint32_t scale_mantissa_bits(const AttentionParams& P) { return __float_as_uint(P.scale_mantissa) & 0x7FFFFFu; }
__device__ __forceinline__ float logit_factor(const AttentionParams& P, int e) { return __uint_as_float(__float_as_uint(logit_power(P, e)) | scale_mantissa_bits(P)); }

// Weights are 2^(logit - unit), the largest 2^15, which FP16 has exactly; where a row's logits are mostly below one of them that is the weight that counts (results in FP16 are off
// by 2.3e-4 so, by 3.0e-4 with a whole number for the unit everywhere).  A largest logit that is more than `most` (15 or a little more) above the unit moves it, and gives what sums so far shrink by.
//   The unit is what is subtracted, after its rounding, in weights and in sums alike.  From 2^12 on it is a whole number that makes the largest weight 2^14 .. 2^15: the rounding of
// logit - 15 would move it further and further, from 2^24 on beyond FP16 or to nothing.  From 2^23 on, where logits are whole numbers, it is the logit.
//   The product is not rounded in a weight's exponent, factor * product - unit, the largest logit is: from kFarLogit on, where that is 2^-5 and more, products have to be rounded as well, or exact.
constexpr float kFarLogit = 524288.0f;
__device__ __forceinline__ bool above_unit(float unit, float largest, float most) { return largest - unit > most; }           // not where both are -infinity
__device__ __forceinline__ float move_unit(float& unit, float largest, float most)
{
    if (!above_unit(unit, largest, most)) return 1.0f;
    const float whole = ceilf(largest), to = fabsf(largest) < 4096.0f ? largest - 15.0f : fabsf(whole) < 8388608.0f ? whole - 15.0f : whole;
    const float shrink = exp2_fast(unit - to);
    unit = to;
    return shrink;
}

}  // namespace zc
