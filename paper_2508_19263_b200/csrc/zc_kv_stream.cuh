// Attention of a few rows over a long cache: the cache's bytes bound it.
//
// Columns: the rows of a sequence times the query heads that share a head of the cache; kCols of them make an item with that head.  A step
// is 64 tokens (32 where they are 128 bytes) of an item.  All steps of a call, in order, are cut into as many equal runs as there are warps on the GPU; a warp goes
// through its run by itself: copies, two barriers, matrix instructions, running maximum and sum, nothing shared with other warps until its end.  So long
// sequences are split, short ones are not, and nobody waits for the longest.  An item that lies in one run is finished by its warp; the
// parts of the others are joined, in order, first in the block, then, where an item goes on in the next block, by a second kernel.
//
// Mathematics of a step, for m16n8k16 instructions on FP16 with FP32 sums: S^T = K Q^T with 16 tokens as rows and 8 columns; then
// O^T += V^T P^T with 16 of the head's width as rows, 16 tokens as the sum's axis.  Both operands from the cache come out of shared memory
// as they are, by ldmatrix (transposed for V), and become FP16 in registers (one conversion for two elements, exact).  The order in which the
// sum over a head's width goes is free, so Q is laid out in the order in which ldmatrix gives K's nibbles.
//   Keys' scales multiply the FP32 sums of each 32 products, values' scales the weights: a block of 32 of the head's width has weights of its own,
// 2^(s - R) times the softmax's, R the largest scale byte that the item's run has met.  So elements go into the products as they are.  Keys' scales are taken over 2^0, and
// over the largest that the run has met from the first of 2^65 or more on, or where queries and scale are far from 1: products, or what makes logits of them, could be
// beyond FP32 where the logits are not.
//   Queries become FP16 over a power of two that brings the row's largest to 2^14 .. 2^15: BF16's eight bits are kept down to 2^-31 of it.
//   Weights are 2^(x - u), u so that the largest is 2^15, in FP32 for the sum, rounded to FP16 for the product with V: off by at most 2^-12 of it
// where it is above 2^-29 of the largest (the scale's power of two counted in), by 2^-40 of the largest below; where logits pass 2^12, 2^-28 and 2^-39.
//   Measured: one token for 64 sequences of 2200 to 8200 tokens, 32 heads of queries over 8 in FP4: 109 us, 3.6 TB/s; the copies alone take 79 us, what is left are the
// conversions' instructions: 630 for 32 tokens, of them 130 conversions and about 100 that bring a conversion its byte, at three warps a scheduler.  A call's
// fixed part is 14 us (one sequence of 4096 tokens): a chain of reads (lengths, pages, elements), one step, joins in the block and between blocks.
//   16 warps with 128 registers: 162 us (spills), 8 with 255: 121; elements scaled one by one instead of sums and weights: 119; 32 tokens a step: 119.  In E4M3 with heads of
// 128 the registers do not quite suffice: 8 bytes a thread are spilled by the 12 warps, 28 by the 8; nothing is in the other shapes.
#pragma once
#include <type_traits>

#include "zc_kv_attention.cuh"

namespace zc {

template <bool FP4_, uint32_t DIM_, uint32_t NT_>
struct StreamShape {
    static constexpr bool kFp4 = FP4_;
    static constexpr uint32_t kDim = DIM_, kNt = NT_, kCols = 8 * NT_;
    static constexpr uint32_t kRow = kFp4 ? kDim / 2 : kDim;               // bytes of a token's head
    static constexpr uint32_t kBlocks = kDim / kKvBlock, kChunks = kRow / 16;
    // Tokens of a step.  What a step costs whatever its tokens (copies, barrier, maxima over the warp) is a third of it at 32.
    static constexpr uint32_t kStep = kRow == 128 ? 32 : 64, kOwn = kStep / 32, kGroups = kStep / 16;
    static constexpr uint32_t kTile = kStep * kRow;                          // keys or values of a step
    static constexpr uint32_t kStage = 2 * kTile, kScales = kStep * kBlocks;
    static constexpr uint32_t kTiles = kDim / 16;                            // of 16 of the head's width
    // 12 warps of 168 registers where 8 columns are all, 8 of 255 for 16
    static constexpr uint32_t kWarps = NT_ == 1 ? 12 : 8, kStages = kRow == 32 ? 3 : 2;
    using Place = Cursor<kCols, kStep>;
    // a part: means of values [kCols][kDim + 4] (the padding spreads lanes over the banks), what weights are over [kCols], sums of weights [kCols]
    static constexpr uint32_t kPartLd = kDim + 4, kPart = kCols * (kPartLd + 2);
    // shared memory of a warp
    static constexpr uint32_t kRing = kStages * kStage, kRingScales = kStages * 2 * kScales;
    static constexpr uint32_t kFactors = kStep * kBlocks * 4;                // of keys (FP32), then of values (FP16, twice)
    // logits of 16 tokens, a lane's four a piece of 16 bytes: where their keys were, if they fit there
    static constexpr bool kLogitsOver = 16 * kRow >= kNt * 512;
    static constexpr uint32_t kLogitsLd = kLogitsOver ? 16 * kRow : kNt * 512;
    static constexpr uint32_t kWarpBytes = kRing + kRingScales + kFactors + (kLogitsOver ? 0 : kGroups * kLogitsLd);
    static constexpr uint32_t kSmem = kWarps * kWarpBytes + 1024;
    static_assert(kWarps <= 16, "a lane for each part of a block");
    static_assert(kPart * 4 <= kRing, "a run's last part goes where its copies were");
    static_assert(kSmem <= kMaxSmem - 2048, "shared memory");
};

// Where the run-th of `runs` equal shares begins.
__device__ __forceinline__ unsigned long long share(unsigned long long total, uint32_t run, uint32_t runs)
{
    // Below 2^63: 2^49 steps in 2^13 runs.  Divided 32 bits at a time, runs being below 2^16: with a division of 64 bits in it the kernel of many rows takes
    // 1400 us where it takes 1280 so (2048 rows over 34816 tokens).
    const unsigned long long all = total * run;
    const uint32_t hi = (uint32_t)(all >> 32), lo = (uint32_t)all, q0 = hi / runs, x1 = (hi - q0 * runs) << 16 | lo >> 16, q1 = x1 / runs, x2 = (x1 - q1 * runs) << 16 | (lo & 0xFFFFu);
    return ((unsigned long long)q0 << 32) + ((unsigned long long)q1 << 16) + x2 / runs;
}

// How many of `blocks` get steps where each takes `least` if it can.
__device__ __forceinline__ uint32_t working_blocks(unsigned long long total, uint32_t least, uint32_t blocks)
{
    return total >= (unsigned long long)least * blocks ? blocks : total ? ((uint32_t)total + least - 1) / least : 1;
}

// A part of an item that a warp leaves to the block.
struct StreamEntry {
    unsigned long long from, to;           // the item's steps among all
    ItemColumns columns;
    uint32_t there;
};

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t w[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t w[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v)
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t mul_half2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// Where the copies put 16 bytes of a row: the swizzle as wide as a row, which spreads eight rows' pieces over all banks.
template <uint32_t ROW>
__device__ __forceinline__ uint32_t swizzled(uint32_t row, uint32_t chunk)
{
    return row * ROW + ((chunk ^ (ROW == 128 ? row & 7 : ROW == 64 ? (row >> 1) & 3 : (row >> 2) & 1)) << 4);
}
// Two tokens' elements of the cache, 16 bits each (the first token's in the low half), as pairs (first, second) of FP16: 4 in FP4, 2 in E4M3.
__device__ __forceinline__ void pairs_fp4(uint32_t w, uint32_t h[4])
{
    uint32_t even, odd;                                                       // byte 0: nibble 0 of both, byte 1: nibble 2; byte 2: nibble 1, byte 3: nibble 3
    asm("lop3.b32 %0, %1, %2, 0x0F0F0F0F, 0xE4;" : "=r"(even) : "r"(w), "r"(w >> 12));         // the mask's bits of the first, the others of the second
    asm("lop3.b32 %0, %1, %2, 0x0F0F0F0F, 0xD8;" : "=r"(odd) : "r"(w), "r"(w << 12));          // the other way round
    asm("{\n\t.reg .b8 b0, b1, b2, b3, c0, c1, c2, c3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\tmov.b32 {c0, c1, c2, c3}, %5;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, c2;\n\tcvt.rn.f16x2.e2m1x2 %2, b1;\n\tcvt.rn.f16x2.e2m1x2 %3, c3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(even), "r"(odd));
}
__device__ __forceinline__ void pairs_e4m3(uint32_t w, uint32_t h[2]) { e4m3_to_half(__byte_perm(w, 0, 0x3120), h); }

// D = A B for m16n8k16; `zero` holds zeros
__device__ __forceinline__ void mma_f16_first(float c[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, const float zero[4])
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(zero[0]), "f"(zero[1]), "f"(zero[2]), "f"(zero[3]));
}
// The largest of a lane's scale bytes, NaN (255) left out.  A word has four bytes, or two in its low half.
template <bool FOUR, uint32_t N>
__device__ __forceinline__ uint32_t largest_scale(const uint32_t (&w)[N])
{
    uint32_t most = 0;
#pragma unroll
    for (uint32_t j = 0; j < N; ++j)
#pragma unroll
        for (uint32_t k = 0; k < (FOUR ? 4 : 2); ++k)
            if (((w[j] >> (8 * k)) & 0xFF) != 255) most = max(most, (w[j] >> (8 * k)) & 0xFF);
    return most;
}
// (1 + mantissa / 2^23) 2^(s - ref) in FP32, s <= ref; NaN for 255.
__device__ __forceinline__ uint32_t key_factor(uint32_t s, uint32_t ref, uint32_t mantissa)
{
    const int e = (int)s - (int)ref + 127;
    return s == 255 ? 0x7FFFFFFFu : e > 0 ? (uint32_t)e << 23 | mantissa : (0x800000u | mantissa) >> min(1 - e, 31);
}
// 2^(s - ref) in FP16, s <= ref; NaN for 255.
__device__ __forceinline__ uint32_t value_factor(uint32_t s, uint32_t ref)
{
    const int e = (int)s - (int)ref + 15;
    return s == 255 ? 0x7E00u : e > 0 ? (uint32_t)e << 10 : 0x400u >> min(1 - e, 31);
}

// Query of a column in the order of the keys' elements in a lane's registers, in FP16 times 2^lift, with the scale's sign.
template <typename S>
__device__ __forceinline__ void load_queries(const AttentionParams& P, const typename S::Place& c, uint32_t col, uint32_t i, uint32_t q[S::kDim / 8], int& lift)
{
#pragma unroll
    for (uint32_t k = 0; k < S::kDim / 8; ++k) q[k] = 0;
    float most = 0.0f;
    if (c.has(P, col)) {
        const uint8_t* p = c.query(P, col);
#pragma unroll
        for (uint32_t k = 0; k < S::kDim / 16; ++k) {
            const uint32_t d = 32 * (k / 2) + (S::kFp4 ? 8 * i + 4 * (k & 1) : 16 * (k & 1) + 4 * i);
            const uint2 w = query_four(P, p + 2 * d);
            q[2 * k] = w.x;
            q[2 * k + 1] = w.y;
        }
#pragma unroll
        for (uint32_t k = 0; k < S::kDim / 8; ++k) {
            const float2 f = query_pair(P, q[k]);
            most = fmaxf(most, fmaxf(fabsf(f.x), fabsf(f.y)));
        }
    }
    most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
    most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
    lift = query_lift(most);
    const float up = copysignf(power_of_two(lift), P.scale_mantissa);
#pragma unroll
    for (uint32_t j = 0; j < S::kDim / 8; ++j) {
        const float2 f = query_pair(P, q[j]);
        q[j] = pack_half(f.x * up, f.y * up);
    }
}
template <typename S>
__device__ __forceinline__ float* partial_of(const AttentionParams& P, uint32_t blocks, uint32_t block, uint32_t slot)
{
    return reinterpret_cast<float*>(P.workspace + ((size_t)blocks * sizeof(BlockEnd) + 255) / 256 * 256) + (size_t)(2 * block + slot) * (S::kCols * (S::kDim + 2));
}
template <typename S>
__device__ __forceinline__ float* part_in_workspace(const AttentionParams& P, uint32_t warp)
{
    return partial_of<S>(P, gridDim.x, gridDim.x, 0) + (size_t)warp * S::kPart;
}
// The joined means of a column whose parts begin at part(k), 0 <= k < count, all lanes together: a lane has kDim / 32 neighbours.  Parts hold means, not
// sums, and are joined with shares that add up to 1: a sum may be beyond FP32 where the mean is not.
// `at` and `weights` say where in a part that which weights are over and the sum of weights of the column are, `means` where its means begin.
template <typename S, typename PART>
__device__ __forceinline__ void join_parts(uint32_t count, PART part, uint32_t means, uint32_t at, uint32_t weights, float v[S::kDim / 32], float& best, float& weight)
{
    constexpr uint32_t N = S::kDim / 32;
    const uint32_t lane = threadIdx.x & 31;
    best = -INFINITY;
    weight = 0.0f;
#pragma unroll
    for (uint32_t n = 0; n < N; ++n) v[n] = 0.0f;
    for (uint32_t k0 = 0; k0 < count; k0 += 32) {
        // a lane has a part
        const float* mine = k0 + lane < count ? part(k0 + lane) : nullptr;
        const uint32_t some = min(32u, count - k0);
        constexpr uint32_t kAtOnce = 16;                       // reads under way
        float x[kAtOnce][N];
        auto read = [&](uint32_t k1) {
#pragma unroll
            for (uint32_t k = 0; k < kAtOnce; ++k) {
                const float* p = reinterpret_cast<const float*>(__shfl_sync(0xFFFFFFFFu, reinterpret_cast<unsigned long long>(mine), (k1 + k) & 31)) + means + lane * N;
                if (k1 + k >= some) continue;
                if (N == 4) { const float4 y = *reinterpret_cast<const float4*>(p); x[k][0] = y.x; x[k][1] = y.y; x[k][N - 2] = y.z; x[k][N - 1] = y.w; }
                else { const float2 y = *reinterpret_cast<const float2*>(p); x[k][0] = y.x; x[k][1] = y.y; }
            }
        };
        read(0);
        const float t = mine ? mine[at] : -INFINITY, w = mine ? mine[weights] : 0.0f;
        float next = t;
        for (int d = 16; d; d >>= 1) next = fmaxf(next, __shfl_xor_sync(0xFFFFFFFFu, next, d));
        next = fmaxf(next, best);
        const float off = next == -INFINITY ? 0.0f : next, old = weight * exp2_fast(best - off), now = w * exp2_fast(t - off);
        best = next;
        float sum = now;
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
        weight = old + sum;
        const float norm = inverse_weight(weight), share = now * norm;
#pragma unroll
        for (uint32_t n = 0; n < N; ++n) v[n] *= old * norm;
        for (uint32_t k1 = 0; k1 < some; k1 += kAtOnce) {
            if (k1) read(k1);
#pragma unroll
            for (uint32_t k = 0; k < kAtOnce; ++k) {
                const float f = __shfl_sync(0xFFFFFFFFu, share, (k1 + k) & 31);
                if (k1 + k < some)
#pragma unroll
                    for (uint32_t n = 0; n < N; ++n) v[n] = fmaf(x[k][n], f, v[n]);
            }
        }
    }
}

template <typename S>
__global__ void __launch_bounds__(S::kWarps * 32, 1) kv_stream_kernel(const AttentionParams P, const __grid_constant__ CUtensorMap key_map, const __grid_constant__ CUtensorMap value_map)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ __align__(8) uint64_t s_full[S::kWarps * S::kStages];
    __shared__ unsigned long long s_cost[ZC_KV_MAX_SEQS / 32];
    __shared__ StreamEntry s_entry[S::kWarps * 2];
    __shared__ uint8_t s_order[S::kWarps][32];
    __shared__ int8_t s_lift[S::kWarps][S::kCols];        // queries are over 2^-lift
    __shared__ volatile uint32_t s_failed;
    constexpr uint32_t kAll = 0xFFFFFFFFu;
    const uint32_t lane = threadIdx.x & 31, warp = warp_index(), g = lane >> 2, i = lane & 3;
    // the swizzle goes by address bits: the rings begin on 1024 bytes
    const uint32_t base = (smem_u32(smem) + 1023) & ~1023u;
    const uint32_t ring = base + warp * S::kRing, rest = base + S::kWarps * S::kRing + warp * (S::kWarpBytes - S::kRing);
    const uint32_t ring_scales = rest, factors = rest + S::kRingScales;
    const uint32_t bars = smem_u32(s_full) + warp * S::kStages * 8;
    if (lane < S::kStages) bar_init(bars + 8 * lane, 1);
    if (lane < 2) s_entry[2 * warp + lane].there = 0;
    if (threadIdx.x == 0) {
        s_failed = 0;
        prefetch_map(&key_map);
        prefetch_map(&value_map);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    grid_wait();
    grid_launch_dependents();

    // ---- which steps are this warp's ----
    const uint32_t chunks = (P.B.n_seqs + 31) / 32;
    SeqSpan span = stream_span<S::kCols, S::kStep>(P, lane);
    unsigned long long total = 0, before = 0, cost = span.cost(P.C.heads);
    if (chunks > 1) {
        for (uint32_t c = warp; c < chunks; c += S::kWarps) {
            unsigned long long sum = stream_span<S::kCols, S::kStep>(P, 32 * c + lane).cost(P.C.heads);
            for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(kAll, sum, d);
            if (lane == 0) s_cost[c] = sum;
        }
        __syncthreads();
        for (uint32_t c = lane; c < chunks; c += 32) total += s_cost[c];
    } else {
        total = cost;
        __syncthreads();
    }
    for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(kAll, total, d);
    // with fewer steps than warps only so many blocks as have a step for each warp: parts of an item are joined in a block rather than between blocks
    const uint32_t blocks = working_blocks(total, S::kWarps, gridDim.x), runs = blocks * S::kWarps, run = blockIdx.x * S::kWarps + warp;
    const bool works = blockIdx.x < blocks;
    const unsigned long long from = works ? share(total, run, runs) : 0, to = works ? share(total, run + 1, runs) : 0;
    const unsigned long long block_from = works ? share(total, blockIdx.x, blocks) : 0, block_to = works ? share(total, blockIdx.x + 1, blocks) : 0;

    // ---- the place of step `from`: sequence, item of the sequence, step of the item ----
    uint32_t b = 0, item = 0, step = 0;
    unsigned long long item_from = 0;                     // the present item's first step among all
    if (from < to) {
        uint32_t c = 0;
        if (chunks > 1) {
            while (before + s_cost[c] <= from) before += s_cost[c++];
            span = stream_span<S::kCols, S::kStep>(P, 32 * c + lane);
            cost = span.cost(P.C.heads);
        }
        unsigned long long upto = cost;                  // inclusive sums over the lanes
        for (int d = 1; d < 32; d <<= 1) {
            const unsigned long long o = __shfl_up_sync(kAll, upto, d);
            if ((int)lane >= d) upto += o;
        }
        const uint32_t k = __ffs(__ballot_sync(kAll, before + upto > from)) - 1;
        b = 32 * c + k;
        const unsigned long long inside = from - before - __shfl_sync(kAll, upto - cost, k);
        const uint32_t steps = __shfl_sync(kAll, span.steps, k);
        item = (uint32_t)(inside >> 32 ? inside / steps : (uint32_t)inside / steps);
        step = (uint32_t)(inside - (unsigned long long)item * steps);
        item_from = from - step;
    }

    // ---- copies: one cursor runs ahead ----
    const KvWaiter wait{P.spin_limit, smem_u32(const_cast<uint32_t*>(&s_failed))};
    typename S::Place ahead;
    ahead.set(span, b, item, step);
    SeqSpan at_span = span;                              // `ahead` may come to the next 32 sequences before
    // the first item's queries are on their way while its pages are looked up
    if (from < to) {
#pragma unroll
        for (uint32_t t = 0; t < S::kNt; ++t) {
            const uint32_t col = ahead.tile * S::kCols + 8 * t + g;
            if (ahead.has(P, col)) asm volatile("prefetch.global.L1 [%0];" :: "l"(ahead.query(P, col) + i * (S::kDim / 2)));
        }
    }
    uint32_t place_base = 0xFFFFFFFFu, place_seq = 0xFFFFFFFFu;
    int pages = 0;
    uint32_t missing = 0;                                 // kGroups bits a stage: groups of 16 tokens that have no page
    const bool endless = (to - from) >> 32 != 0;          // five hours at 4 us a step: not begun
    const uint32_t count = endless ? 0u : (uint32_t)(to - from);
    if (endless) wait.give_up();
    uint32_t sent = 0;
    const uint32_t piece_tokens = min(1u << P.C.page_shift, S::kStep), pieces = S::kStep / piece_tokens;
    auto send = [&](uint32_t st) {
        // the pages of the next 32 places are kept in the lanes
        const uint32_t t0 = ahead.token(), place = t0 >> P.C.page_shift;
        if (place - place_base >= 32 || place_seq != ahead.b) {
            place_base = place & ~31u;
            place_seq = ahead.b;
            const uint32_t mine = place_base + lane;
            pages = mine < P.B.max_pages && (mine << P.C.page_shift) < (uint32_t)ahead.to && ((mine + 1) << P.C.page_shift) > (uint32_t)ahead.from ? kv_page(P.C, P.B, ahead.b, mine) : -1;
        }
        const uint32_t bar = bars + 8 * st, to_keys = ring + st * S::kStage, to_scales = ring_scales + st * 2 * S::kScales;
        const uint32_t there = __ballot_sync(kAll, pages >= 0) >> (place & 31), have = there & ((1u << pieces) - 1);
        if (elect_one()) bar_expect(bar, __popc(have) * piece_tokens * 2 * (S::kRow + S::kBlocks));
        missing &= ~(((1u << S::kGroups) - 1) << (S::kGroups * st));
        for (uint32_t k = 0; k < pieces; ++k) {
            const int page = __shfl_sync(kAll, pages, (place + k) & 31);
            const uint32_t at = k * piece_tokens;
            if (page < 0) {
                missing |= ((1u << (piece_tokens / 16)) - 1) << (S::kGroups * st + at / 16);
                continue;
            }
            const uint32_t row = (((uint32_t)page * P.C.heads + ahead.head) << P.C.page_shift) + (t0 & ((1u << P.C.page_shift) - 1));
            if (!P.skip_copy && elect_one()) {
                tensor_copy<1>(to_keys + at * S::kRow, &key_map, 0, (int)row, bar);
                tensor_copy<1>(to_keys + S::kTile + at * S::kRow, &value_map, 0, (int)row, bar);
                bulk_copy(to_scales + at * S::kBlocks, P.C.scales[0] + (uint64_t)row * S::kBlocks, piece_tokens * S::kBlocks, bar);
                bulk_copy(to_scales + S::kScales + at * S::kBlocks, P.C.scales[1] + (uint64_t)row * S::kBlocks, piece_tokens * S::kBlocks, bar);
            }
        }
        __syncwarp();
        ahead.next(P, span);
        ++sent;
    };
#pragma unroll
    for (uint32_t st = 0; st < S::kStages; ++st)
        if (sent < count) send(st);

    // ---- the steps ----
    typename S::Place at;
    at.set(at_span, b, item, step);
    float acc[S::kNt][S::kTiles][4], top[S::kNt][2], sum[S::kNt][2], factor[S::kNt][2];
    uint32_t q[S::kNt][S::kDim / 8];
    int lo[S::kNt][2], hi[S::kNt][2], lo_most = 0, hi_least = 0;
    // where a lane's rows for ldmatrix begin: swizzled by the lane alone, 16 tokens further the same
    uint32_t key_at[S::kChunks / 2], value_at[S::kChunks / 2];
#pragma unroll
    for (uint32_t c = 0; c < S::kChunks; c += 2) {
        key_at[c / 2] = swizzled<S::kRow>((lane & 7) + 8 * ((lane >> 3) & 1), c + (lane >> 4));
        value_at[c / 2] = swizzled<S::kRow>((lane & 7) + 8 * (lane >> 4), c + ((lane >> 3) & 1));
    }
    float zero[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) asm volatile("mov.b32 %0, 0;" : "=f"(zero[k]));
    uint32_t ref = 0, key_ref = 0;                       // scale bytes that values' and keys' scales are over
    bool fresh = true, ok = !endless, careful = false;       // careful: key_ref is the largest so far, else 127
    auto set_factors = [&]() {
#pragma unroll
        for (uint32_t t = 0; t < S::kNt; ++t) {
            const float own = logit_power(P, (int)key_ref - 127 - s_lift[warp][8 * t + g]);
            factor[t][0] = __shfl_sync(kAll, own, 8 * i);
            factor[t][1] = __shfl_sync(kAll, own, 8 * i + 4);
        }
    };
    uint32_t st = 0, parity = 0;
    for (uint32_t done = 0; done < count; ++done) {
        if (fresh) {
            // the item's columns: queries, limits
            fresh = false;
            ref = 0;
            careful = false;
            lo_most = 0;
            hi_least = 0x7FFFFFFF;
#pragma unroll
            for (uint32_t t = 0; t < S::kNt; ++t) {
                int lift;
                load_queries<S>(P, at, at.tile * S::kCols + 8 * t + g, i, q[t], lift);
                if (i == 0) s_lift[warp][8 * t + g] = (int8_t)lift;
                careful |= abs(P.scale_exponent - lift) > 100;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t col = at.tile * S::kCols + 8 * t + 2 * i + k;
                    at.column_limits(P, col, lo[t][k], hi[t][k]);
                    lo_most = max(lo_most, lo[t][k]);
                    hi_least = min(hi_least, hi[t][k]);
                    top[t][k] = -INFINITY;
                    sum[t][k] = 0.0f;
                }
#pragma unroll
                for (uint32_t m = 0; m < S::kTiles; ++m)
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[t][m][k] = 0.0f;
            }
            careful = __any_sync(kAll, careful);
            __syncwarp();
            key_ref = careful ? 0 : 127;
            set_factors();
            lo_most = __reduce_max_sync(kAll, lo_most);
            hi_least = __reduce_min_sync(kAll, hi_least);
        }
        if (!wait.warp(bars + 8 * st, parity)) { ok = false; break; }
        const uint32_t keys = ring + st * S::kStage, values = keys + S::kTile, scales = ring_scales + st * 2 * S::kScales;
        const uint32_t logits = S::kLogitsOver ? keys : factors + S::kFactors;
        const int t0 = (int)at.token();
        const uint32_t gone = (missing >> (S::kGroups * st)) & ((1u << S::kGroups) - 1);
        const bool plain = t0 >= lo_most && t0 + (int)S::kStep <= hi_least && gone == 0;

        // scales: a lane has every 32nd token
        uint32_t ks[S::kOwn], vs[S::kOwn], hidden = 0, poisoned[S::kOwn] = {};     // poisoned: tokens with NaN in their values that not every column sees
#pragma unroll
        for (uint32_t j = 0; j < S::kOwn; ++j) {
            if (S::kBlocks == 4) { ks[j] = lds32(scales + 4 * (32 * j + lane)); vs[j] = lds32(scales + S::kScales + 4 * (32 * j + lane)); }
            else { ks[j] = lds16(scales + 2 * (32 * j + lane)); vs[j] = lds16(scales + S::kScales + 2 * (32 * j + lane)); }
        }
        if (!plain) {
#pragma unroll
            for (uint32_t j = 0; j < S::kOwn; ++j) {
                const uint32_t r = 32 * j + lane;
                const int t = t0 + (int)r;
                bool hide = t < at.from || t >= at.to || (gone >> (r >> 4)) & 1, nan = false;
#pragma unroll
                for (uint32_t k = 0; k < S::kBlocks; ++k) nan |= ((vs[j] >> (8 * k)) & 0xFF) == 255;
                if (!S::kFp4) {
#pragma unroll
                    for (uint32_t c = 0; c < S::kChunks; ++c) {
                        const uint4 w = lds128(values + swizzled<S::kRow>(r, c));
                        nan |= nan_bytes(w.x) || nan_bytes(w.y) || nan_bytes(w.z) || nan_bytes(w.w);
                    }
                }
                nan = nan && !hide && !(t >= lo_most && t < hi_least);
                poisoned[j] = __ballot_sync(kAll, nan);
                hide |= nan;
                if (hide) {
                    hidden |= 1u << j;
                    ks[j] = vs[j] = 0;
                    if (!S::kFp4) {
                        const uint32_t none[4] = {};
#pragma unroll
                        for (uint32_t c = 0; c < S::kChunks; ++c) sts128(values + swizzled<S::kRow>(r, c), none);
                        fence_async_shared();            // the next copy comes here
                    }
                }
            }
        }
        {
            // keys' scales times the mantissa of the call's, [token][block] in FP32: what is left of `factor` is a power of two
            const uint32_t mantissa = scale_mantissa_bits(P);
            uint32_t big = 0;                            // of 192 or more
#pragma unroll
            for (uint32_t j = 0; j < S::kOwn; ++j) {
                uint32_t f[4];
                big |= ks[j] & (ks[j] << 1) & 0x80808080u;
#pragma unroll
                for (uint32_t k = 0; k < S::kBlocks; ++k) f[k] = max((k < 3 ? ks[j] << (k < 3 ? 23 - 8 * k : 0) : ks[j] >> 1) & 0x7F800000u | mantissa, 0x00400000u | mantissa >> 1);       // the latter for 2^-127
                if (S::kBlocks == 4) sts128(factors + 16 * (32 * j + lane), f);
                else sts64(factors + 8 * (32 * j + lane), f[0], f[1]);
            }
            careful = __any_sync(kAll, careful || big);
            if (careful) {
                key_ref = max(key_ref, __reduce_max_sync(kAll, largest_scale<S::kBlocks == 4>(ks)));
                set_factors();
#pragma unroll 1
                for (uint32_t k = 0; k < S::kOwn * S::kBlocks; ++k) {
                    const uint32_t j = k / S::kBlocks, b = k % S::kBlocks, w = j ? ks[S::kOwn - 1] : ks[0];
                    sts_f1(factors + 4 * (S::kBlocks * (32 * j + lane) + b), __uint_as_float(key_factor((w >> (8 * b)) & 0xFF, key_ref, mantissa)));
                }
            }
            __syncwarp();
        }

        // logits, 16 tokens at a time: rows g and g + 8, columns 2i and 2i + 1.  They wait for the step's maximum where their keys were.
        float best[S::kNt][2];
#pragma unroll
        for (uint32_t t = 0; t < S::kNt; ++t) best[t][0] = best[t][1] = -INFINITY;
#pragma unroll 2
        for (uint32_t m = 0; m < S::kGroups; ++m) {
            float f[2][4], p[S::kNt][4];
            const uint32_t row = 16 * m + g;
            if (S::kBlocks == 4) { lds_f4(factors + 16 * row, f[0]); lds_f4(factors + 16 * (row + 8), f[1]); }
            else { lds_f2(factors + 8 * row, f[0]); lds_f2(factors + 8 * (row + 8), f[1]); }
#pragma unroll
            for (uint32_t t = 0; t < S::kNt; ++t)
#pragma unroll
                for (int k = 0; k < 4; ++k) p[t][k] = 0.0f;
#pragma unroll
            for (uint32_t c = 0; c < S::kChunks; c += 2) {
                uint32_t w[4];
                ldmatrix4(keys + m * (16 * S::kRow) + key_at[c / 2], w);
#pragma unroll
                for (uint32_t h = 0; h < (S::kFp4 ? 2 : 1); ++h) {
                    uint32_t a[8];                       // rows g, g + 8 of the first four pairs, then of the next
                    if (S::kFp4) {
                        uint32_t x[4], y[4];
                        fp4_to_half(w[2 * h], x);
                        fp4_to_half(w[2 * h + 1], y);
#pragma unroll
                        for (int k = 0; k < 4; ++k) { a[2 * k] = x[k]; a[2 * k + 1] = y[k]; }
                    } else {
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            uint32_t x[2], y[2];
                            e4m3_to_half(w[2 * k], x);
                            e4m3_to_half(w[2 * k + 1], y);
                            a[4 * k] = x[0]; a[4 * k + 1] = y[0]; a[4 * k + 2] = x[1]; a[4 * k + 3] = y[1];
                        }
                    }
                    const uint32_t block = S::kFp4 ? c + h : c / 2;
#pragma unroll
                    for (uint32_t t = 0; t < S::kNt; ++t) {
                        float d[4];
                        mma_f16_first(d, a[0], a[1], a[2], a[3], q[t][4 * block], q[t][4 * block + 1], zero);
                        mma_f16(d, a[4], a[5], a[6], a[7], q[t][4 * block + 2], q[t][4 * block + 3]);
                        p[t][0] = fmaf(d[0], f[0][block], p[t][0]);
                        p[t][1] = fmaf(d[1], f[0][block], p[t][1]);
                        p[t][2] = fmaf(d[2], f[1][block], p[t][2]);
                        p[t][3] = fmaf(d[3], f[1][block], p[t][3]);
                    }
                }
            }
            __syncwarp();
#pragma unroll
            for (uint32_t t = 0; t < S::kNt; ++t) {
                best[t][0] = fmaxf(best[t][0], fmaxf(p[t][0], p[t][2]));
                best[t][1] = fmaxf(best[t][1], fmaxf(p[t][1], p[t][3]));
                sts_f4(logits + (m * S::kLogitsLd + t * 512) + 16 * lane, p[t]);
            }
        }

        if (!plain) {
            // what a column does not see
#pragma unroll
            for (uint32_t t = 0; t < S::kNt; ++t) {
                best[t][0] = best[t][1] = -INFINITY;
#pragma unroll 1
                for (uint32_t m = 0; m < S::kGroups; ++m) {
                    const uint32_t nan = (m < 2 ? poisoned[0] : poisoned[S::kOwn - 1]) >> (16 * (m & 1)), where = logits + (m * S::kLogitsLd + t * 512) + 16 * lane;
                    float p[4];
                    lds_f4(where, p);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t r = g + 8 * (k >> 1);
                        const int tok = t0 + (int)(16 * m + r);
                        const bool seen = tok >= lo[t][k & 1] && tok < hi[t][k & 1] && !((gone >> m) & 1);
                        if ((nan >> r) & 1) p[k] = __int_as_float(0x7FFFFFFF);
                        if (!seen) p[k] = -INFINITY;
                        best[t][k & 1] = fmaxf(best[t][k & 1], p[k]);
                    }
                    sts_f4(where, p);
                }
            }
        }

        // what weights are over, after the largest so far
        bool above = false;
        float off[S::kNt][2];
#pragma unroll
        for (uint32_t t = 0; t < S::kNt; ++t)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float x = best[t][k];
                x = fmaxf(x, __shfl_xor_sync(kAll, x, 4));
                x = fmaxf(x, __shfl_xor_sync(kAll, x, 8));
                best[t][k] = fmaxf(x, __shfl_xor_sync(kAll, x, 16)) * factor[t][k];
                above |= above_unit(top[t][k], best[t][k], 15.0f);
            }
        if (__any_sync(kAll, above)) {
#pragma unroll
            for (uint32_t t = 0; t < S::kNt; ++t)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float shrink = move_unit(top[t][k], best[t][k], 15.0f);
                    sum[t][k] *= shrink;
#pragma unroll
                    for (uint32_t m = 0; m < S::kTiles; ++m) {
                        acc[t][m][k] *= shrink;
                        acc[t][m][k + 2] *= shrink;
                    }
                }
        }
#pragma unroll
        for (uint32_t t = 0; t < S::kNt; ++t)
#pragma unroll
            for (int k = 0; k < 2; ++k) off[t][k] = top[t][k] == -INFINITY ? 0.0f : -top[t][k];

        {
            // values' scales over the largest so far, [token][block] in FP16, twice in a word; every lane is done with the keys'
            __syncwarp();
            uint32_t v01[S::kOwn], v23[S::kOwn], mine = 0, least = 255;
            bool odd = false;
#pragma unroll
            for (uint32_t j = 0; j < S::kOwn; ++j) {
                v01[j] = __byte_perm(vs[j], 0, 0x4140);
                v23[j] = S::kBlocks == 4 ? __byte_perm(vs[j], 0, 0x4342) : v01[j];
                const uint32_t most2 = __vmaxu2(v01[j], v23[j]), least2 = __vminu2(v01[j], v23[j]);
                mine = max(mine, max(most2 & 0xFFFFu, most2 >> 16));
                least = min(least, min(least2 & 0xFFFFu, least2 >> 16));
            }
            if (mine == 255) {
                odd = true;
                mine = largest_scale<S::kBlocks == 4>(vs);
            }
            const uint32_t most = __reduce_max_sync(kAll, mine);
            if (most > ref) {
                const float shrink = ldexpf(1.0f, max((int)ref - (int)most, -200));
                ref = most;
#pragma unroll
                for (uint32_t t = 0; t < S::kNt; ++t)
#pragma unroll
                    for (uint32_t m = 0; m < S::kTiles; ++m)
#pragma unroll
                        for (int k = 0; k < 4; ++k) acc[t][m][k] *= shrink;
            }
            const uint32_t off = (ref - 15) * 0x10001u;                       // no half borrows from the other: s + 15 > ref
            const bool quick = !odd && !hidden && least + 14 >= ref;
#pragma unroll
            for (uint32_t j = 0; j < S::kOwn; ++j) {
                uint32_t f[4];
                if (quick) {
                    const uint32_t f01 = (v01[j] - off) << 10, f23 = (v23[j] - off) << 10;
                    f[0] = __byte_perm(f01, 0, 0x1010);
                    f[1] = __byte_perm(f01, 0, 0x3232);
                    f[2] = __byte_perm(f23, 0, 0x1010);
                    f[3] = __byte_perm(f23, 0, 0x3232);
                } else {
#pragma unroll
                    for (uint32_t k = 0; k < S::kBlocks; ++k) f[k] = (hidden >> j) & 1 ? 0u : value_factor((vs[j] >> (8 * k)) & 0xFF, ref) * 0x10001u;
                }
                if (S::kBlocks == 4) sts128(factors + 16 * (32 * j + lane), f);
                else sts64(factors + 8 * (32 * j + lane), f[0], f[1]);
            }
            __syncwarp();
        }

        // weights and weighted values, 16 tokens at a time
#pragma unroll 2
        for (uint32_t m = 0; m < S::kGroups; ++m) {
            uint32_t f[2][4], pb[S::kNt][S::kBlocks][2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {                  // tokens g and g + 8
                const uint32_t where = factors + (16 * m + 8 * k + g) * S::kBlocks * 4;
                if (S::kBlocks == 4) { const uint4 v = lds128(where); f[k][0] = v.x; f[k][1] = v.y; f[k][2] = v.z; f[k][3] = v.w; }
                else lds64(where, f[k][0], f[k][1]);
            }
#pragma unroll
            for (uint32_t t = 0; t < S::kNt; ++t) {
                float p[4];
                lds_f4(logits + (m * S::kLogitsLd + t * 512) + 16 * lane, p);
#pragma unroll
                for (int k = 0; k < 4; ++k) p[k] = exp2_fast(fmaf(p[k], factor[t][k & 1], off[t][k & 1]));
                sum[t][0] += p[0] + p[2];
                sum[t][1] += p[1] + p[3];
                const uint32_t w0 = pack_half(p[0], p[1]), w1 = pack_half(p[2], p[3]);
#pragma unroll
                for (uint32_t k = 0; k < S::kBlocks; ++k) {
                    pb[t][k][0] = transpose8x8(mul_half2(w0, f[0][k]));
                    pb[t][k][1] = transpose8x8(mul_half2(w1, f[1][k]));
                }
            }
#pragma unroll
            for (uint32_t c = 0; c < S::kChunks; c += 2) {
                uint32_t w[4];                             // chunk c, c + 1 of the first eight tokens, then of the next
                ldmatrix4_trans(values + m * (16 * S::kRow) + value_at[c / 2], w);
#pragma unroll
                for (uint32_t h = 0; h < 2; ++h) {
                    const uint32_t block = S::kFp4 ? c + h : c / 2;
                    constexpr uint32_t kPairs = S::kFp4 ? 4 : 2;
                    uint32_t x[4], y[4];
                    if (S::kFp4) { pairs_fp4(w[h], x); pairs_fp4(w[h + 2], y); }
                    else { pairs_e4m3(w[h], x); pairs_e4m3(w[h + 2], y); }
#pragma unroll
                    for (uint32_t u = 0; u < kPairs / 2; ++u)
#pragma unroll
                        for (uint32_t t = 0; t < S::kNt; ++t)
                            mma_f16(acc[t][(c + h) * (kPairs / 2) + u], x[2 * u], x[2 * u + 1], y[2 * u], y[2 * u + 1], pb[t][block][0], pb[t][block][1]);
                }
            }
        }
        if (S::kLogitsOver) fence_async_shared();        // the next copy comes where the logits were
        __syncwarp();                                    // everybody is done with the stage
        const uint32_t used = st;
        if (++st == S::kStages) { st = 0; parity ^= 1; }
        if (sent < count) send(used);

        // the item's, or the run's, end
        const bool item_ends = at.last();
        if (item_ends || done + 1 == count) {
            const unsigned long long item_to = item_from + at.steps;
#pragma unroll
            for (uint32_t t = 0; t < S::kNt; ++t)
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    for (int d = 4; d < 32; d <<= 1) sum[t][k] += __shfl_xor_sync(kAll, sum[t][k], d);
            const bool whole = item_from >= from && item_to <= to;
            const float unit = e8m0_value(ref);
            const uint32_t slot = done + 1 == count ? 1u : 0u;           // the run's last part goes where its copies were, an earlier one (there is one at most) to the workspace
            float* early = part_in_workspace<S>(P, blockIdx.x * S::kWarps + warp);
#pragma unroll
            for (uint32_t t = 0; t < S::kNt; ++t) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t in_tile = 8 * t + 2 * i + k, col = at.tile * S::kCols + in_tile;
                    const float total_weight = sum[t][k], norm = inverse_weight(total_weight);         // before `unit`: the sum itself may be beyond FP32
                    uint8_t* out = nullptr;
                    if (whole && at.has(P, col)) {
                        out = at.out(P, col);
                        if (P.lse && g == 0) P.lse[at.lse(P, col)] = lse_of(top[t][k], total_weight);
                    }
#pragma unroll
                    for (uint32_t m = 0; m < S::kTiles; m += S::kFp4 ? 2 : 1) {
                        constexpr uint32_t kSide = S::kFp4 ? 4 : 2;        // neighbours of the head's width
                        float v[4];
                        v[0] = acc[t][m][k] * norm * unit;
                        v[1] = acc[t][m][k + 2] * norm * unit;
                        if (S::kFp4) {
                            v[2] = acc[t][m + 1][k] * norm * unit;
                            v[3] = acc[t][m + 1][k + 2] * norm * unit;
                        }
                        const uint32_t d = 16 * m + kSide * g;
                        if (out) store_out<kSide>(P, out, d, v);
                        else if (!whole) {
                            if (slot == 0) {
                                for (uint32_t n = 0; n < kSide; ++n) early[in_tile * S::kPartLd + d + n] = v[n];
                            } else if (S::kFp4) sts_f4(ring + (in_tile * S::kPartLd + d) * 4, v);
                            else sts_f2(ring + (in_tile * S::kPartLd + d) * 4, v);
                        }
                    }
                    if (!whole && g == 0) {
                        if (slot == 0) {
                            early[S::kCols * S::kPartLd + in_tile] = top[t][k];
                            early[S::kCols * S::kPartLd + S::kCols + in_tile] = total_weight;
                        } else {
                            sts_f1(ring + (S::kCols * S::kPartLd + in_tile) * 4, top[t][k]);
                            sts_f1(ring + (S::kCols * S::kPartLd + S::kCols + in_tile) * 4, total_weight);
                        }
                    }
                }
            }
            if (!whole && lane == 0) {
                StreamEntry& e = s_entry[2 * warp + slot];
                e.from = item_from;
                e.to = item_to;
                e.columns = at.columns(P);
                e.there = 1;
            }
            item_from = item_to;
            fresh = true;
        }
        at.next(P, at_span);
    }
    if (!ok) {
        // copies under way end, or are waited for as long as anything else, before the block does
        for (uint32_t s = 0; s < S::kStages; ++s)
            if (sent > s) settled(bars + 8 * s, ((sent - 1 - s) / S::kStages) & 1, P.spin_limit);
        if (lane == 0) atomicOr(P.B.marks, kKvGaveUp);
    }
    __syncthreads();
    BlockEnd* ends = reinterpret_cast<BlockEnd*>(P.workspace) + blockIdx.x;
    if (s_failed) {
        if (threadIdx.x == 0) ends->there = 0;
        return;
    }

    // ---- the block's parts, in order: a warp has a column of an item ----
    const uint8_t* rings = smem + (base - smem_u32(smem));
    uint32_t parts = 0;
    {
        const bool there = lane < 2 * S::kWarps && s_entry[lane].there;
        const uint32_t mask = __ballot_sync(kAll, there);
        if (there) s_order[warp][__popc(mask & ((1u << lane) - 1))] = (uint8_t)lane;
        parts = __popc(mask);
        __syncwarp();
    }
    const uint8_t* order = s_order[warp];
    bool goes_on = false;
    uint32_t unit = 0;
    for (uint32_t e = 0; e < parts;) {
        const StreamEntry& entry = s_entry[order[e]];
        const unsigned long long item_at = entry.from, item_to = entry.to;
        uint32_t count = 1;
        while (e + count < parts && s_entry[order[e + count]].from == item_at) ++count;
        const bool begins = item_at >= block_from, whole = begins && item_to <= block_to;
        const ItemColumns columns = entry.columns;
        if (!whole && begins) {
            goes_on = true;
            if (threadIdx.x == 0) *ends = BlockEnd{item_to, total, columns, 1, {}};
        }
        for (uint32_t in_tile = 0; in_tile < columns.count; ++in_tile, ++unit) {
            if (unit % S::kWarps != warp) continue;
            auto part = [&](uint32_t k) -> const float* {
                const uint32_t at = order[e + k];
                return at & 1 ? reinterpret_cast<const float*>(rings + (at >> 1) * S::kRing) : part_in_workspace<S>(P, blockIdx.x * S::kWarps + (at >> 1));
            };
            float v[S::kDim / 32], best, weight;
            join_parts<S>(count, part, in_tile * S::kPartLd, S::kCols * S::kPartLd + in_tile, S::kCols * S::kPartLd + S::kCols + in_tile, v, best, weight);
            constexpr uint32_t N = S::kDim / 32;
            if (whole) finish_column<N>(P, columns, in_tile, lane * N, v, best, weight);
            else {
                float* to_part = partial_of<S>(P, gridDim.x, blockIdx.x, begins ? 1 : 0);
                if (N == 4) *reinterpret_cast<float4*>(to_part + in_tile * S::kDim + lane * N) = make_float4(v[0], v[1], v[N - 2], v[N - 1]);
                else *reinterpret_cast<float2*>(to_part + in_tile * S::kDim + lane * N) = make_float2(v[0], v[1]);
                if (lane == 0) {
                    to_part[S::kCols * S::kDim + in_tile] = best;
                    to_part[S::kCols * S::kDim + S::kCols + in_tile] = weight;
                }
            }
        }
        e += count;
    }
    if (!goes_on && threadIdx.x == 0) ends->there = 0;
}

// The items that go on from one block to the next: blocks for the item that begins and does not end in a block, a warp a column.
template <typename S>
__global__ void __launch_bounds__(256) kv_join_kernel(const AttentionParams P, uint32_t grid, uint32_t least)
{
    grid_wait();
    grid_launch_dependents();
    const BlockEnd end = reinterpret_cast<const BlockEnd*>(P.workspace)[blockIdx.x];
    const uint32_t lane = threadIdx.x & 31;
    if (!end.there) return;
    // up to the last block whose steps begin before the item's end
    const uint32_t blocks = working_blocks(end.total, least, grid);
    const unsigned long long all = end.to * blocks - 1;
    const uint32_t last = all >> 32 ? (uint32_t)(all / end.total) : (uint32_t)all / (uint32_t)end.total, count = last - blockIdx.x + 1;
    auto part = [&](uint32_t k) -> const float* { return partial_of<S>(P, grid, blockIdx.x + k, k == 0 ? 1 : 0); };
    constexpr uint32_t N = S::kDim / 32;
    for (uint32_t in_tile = blockIdx.y * 8 + (threadIdx.x >> 5); in_tile < end.columns.count; in_tile += gridDim.y * 8) {
        float v[N], best, weight;
        join_parts<S>(count, part, in_tile * S::kDim, S::kCols * S::kDim + in_tile, S::kCols * S::kDim + S::kCols + in_tile, v, best, weight);
        finish_column<N>(P, end.columns, in_tile, lane * N, v, best, weight);
    }
}

}  // namespace zc
