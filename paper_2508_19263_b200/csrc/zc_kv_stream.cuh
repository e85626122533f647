// Attention of a few rows over a long cache: the cache's bytes bound it.
//
// Columns: the rows of a sequence times the query heads that share a head of the cache; kCols of them make an item with that head.  A step
// is 32 tokens of an item.  All steps of a call, in order, are cut into as many equal runs as there are warps on the GPU; a warp goes
// through its run by itself: copies, two barriers, matrix instructions, running maximum and sum, nothing shared with other warps until its end.  So long
// sequences are split, short ones are not, and nobody waits for the longest.  An item that lies in one run is finished by its warp; the
// parts of the others are joined, in order, first in the block, then, where an item goes on in the next block, by a second kernel.
//
// Mathematics of a step, for m16n8k16 instructions on FP16 with FP32 sums: S^T = K Q^T with 16 tokens as rows and 8 columns; then
// O^T += V^T P^T with 16 of the head's width as rows, 16 tokens as the sum's axis.  Both operands from the cache come out of shared memory
// as they are, by ldmatrix (transposed for V), and become FP16 in registers (one conversion for two elements, exact).  The order in which the
// sum over a head's width goes is free, so Q is laid out in the order in which ldmatrix gives K's nibbles.
//   Keys' scales multiply the FP32 sums of each 32 products.  Values' scales multiply the elements, as 2^(s - R + kLift) with R the largest scale
// byte that the item's run has met: exact unless a scale is 2^-35 (E4M3: 2^-22) of the largest, and off by at most 2^-25 of a unit that is 2^-kLift of it then.
//   Queries become FP16 over a power of two that brings the row's largest to 2^14 .. 2^15: BF16's eight bits are kept down to 2^-31 of it.
//   Weights are 2^(x - max + 15), in FP32 for the sum, rounded to FP16 for the product with V: off by at most 2^-12 of it where it is above 2^-29 of the
// largest, by 2^-40 of the largest below.
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
    static constexpr uint32_t kTile = kStepTokens * kRow;                    // keys or values of a step
    static constexpr uint32_t kStage = 2 * kTile, kScales = kStepTokens * kBlocks;
    static constexpr uint32_t kTiles = kDim / 16;                            // of 16 of the head's width
    // 16 warps of 128 registers where two stages each and the parts fit into shared memory, else 8 of up to 255
    static constexpr uint32_t kWarps = NT_ == 1 && kRow <= 64 ? 16 : 8;
    static constexpr uint32_t kStages = kRow == 32 ? 4 : NT_ == 2 && kRow == 64 ? 4 : 2;
    static constexpr int kLift = kFp4 ? 12 : 6;                              // 6 * 2^12 and 448 * 2^6 are FP16 numbers
    // a part: sums [kCols][kDim + 4] (the padding spreads lanes over the banks), largest logits [kCols], sums of weights [kCols]
    static constexpr uint32_t kPartLd = kDim + 4, kPart = kCols * (kPartLd + 2);
    // shared memory of a warp
    static constexpr uint32_t kRing = kStages * kStage, kRingScales = kStages * 2 * kScales;
    static constexpr uint32_t kFactors = kStepTokens * kBlocks * 4;          // of keys (FP32); of values (pairs of FP16) half of it
    static constexpr uint32_t kWarpBytes = kRing + kRingScales + kFactors + kFactors / 2 + kPart * 4;
    static constexpr uint32_t kSmem = kWarps * kWarpBytes + 1024;
    static_assert(kPart * 4 <= kRing, "a run's last part goes where its copies were");
    static_assert(kSmem <= kMaxSmem - 2048, "shared memory");
};

// A part of an item that a warp leaves to the block.
struct StreamEntry {
    unsigned long long from, to;           // the item's steps among all
    uint32_t b, item, there;
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
    const uint32_t even = (w & 0x0F0F0F0Fu) | ((w >> 12) & 0xF0F0F0F0u);        // byte 0: nibble 0 of both, byte 1: nibble 2
    const uint32_t odd = (w & 0xF0F0F0F0u) | ((w << 12) & 0x0F0F0F0Fu);         // byte 2: nibble 1 of both, byte 3: nibble 3
    asm("{\n\t.reg .b8 b0, b1, b2, b3, c0, c1, c2, c3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\tmov.b32 {c0, c1, c2, c3}, %5;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, c2;\n\tcvt.rn.f16x2.e2m1x2 %2, b1;\n\tcvt.rn.f16x2.e2m1x2 %3, c3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(even), "r"(odd));
}
__device__ __forceinline__ void pairs_e4m3(uint32_t w, uint32_t h[2]) { e4m3_to_half(__byte_perm(w, 0, 0x3120), h); }

// 2^(s - ref + lift) in FP16; 255 gives NaN.
__device__ __forceinline__ uint32_t value_factor(uint32_t s, uint32_t ref, int lift)
{
    const int e = (int)s - (int)ref + lift + 15;
    return s == 255 ? 0x7E00u : e > 0 ? (uint32_t)e << 10 : 0x400u >> min(1 - e, 31);
}

// Query of a column in the order of the keys' elements in a lane's registers, in FP16 times 2^k; factor: what makes a logit of a product.
template <typename S>
__device__ __forceinline__ void load_queries(const AttentionParams& P, const Cursor<S::kCols>& c, uint32_t col, uint32_t i, uint32_t q[S::kDim / 8], float& factor)
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
    const int k = query_lift(most);
    const float lift = power_of_two(k);
#pragma unroll
    for (uint32_t j = 0; j < S::kDim / 8; ++j) {
        const float2 f = query_pair(P, q[j]);
        q[j] = pack_half(f.x * lift, f.y * lift);
    }
    factor = ldexpf(P.scale_log2, -k);
}
template <typename S>
__device__ __forceinline__ float* partial_of(const AttentionParams& P, uint32_t blocks, uint32_t block, uint32_t slot)
{
    return reinterpret_cast<float*>(P.workspace + ((size_t)blocks * sizeof(BlockEnd) + 255) / 256 * 256) + (size_t)(2 * block + slot) * (S::kCols * (S::kDim + 2));
}
// Where a warp's part lies: its first one in a place of its own, its last one where its copies were.
template <typename S>
__device__ __forceinline__ uint32_t part_of(uint32_t base, uint32_t entry)
{
    const uint32_t warp = entry >> 1;
    return entry & 1 ? base + warp * S::kRing : base + S::kWarps * S::kRing + warp * (S::kWarpBytes - S::kRing) + (S::kWarpBytes - S::kRing - S::kPart * 4);
}

template <typename S>
__global__ void __launch_bounds__(S::kWarps * 32, 1) kv_stream_kernel(const AttentionParams P, const __grid_constant__ CUtensorMap key_map, const __grid_constant__ CUtensorMap value_map)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ __align__(8) uint64_t s_full[S::kWarps * S::kStages];
    __shared__ unsigned long long s_cost[ZC_KV_MAX_SEQS / 32];
    __shared__ StreamEntry s_entry[S::kWarps * 2];
    __shared__ volatile uint32_t s_failed;
    constexpr uint32_t kAll = 0xFFFFFFFFu;
    const uint32_t lane = threadIdx.x & 31, warp = warp_index(), g = lane >> 2, i = lane & 3;
    // the swizzle goes by address bits: the rings begin on 1024 bytes
    const uint32_t base = (smem_u32(smem) + 1023) & ~1023u;
    const uint32_t ring = base + warp * S::kRing, rest = base + S::kWarps * S::kRing + warp * (S::kWarpBytes - S::kRing);
    const uint32_t ring_scales = rest, key_factors = rest + S::kRingScales, value_factors = key_factors + S::kFactors, first_part = value_factors + S::kFactors / 2;
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
    SeqSpan span = stream_span<S::kCols>(P, lane);
    unsigned long long total = 0, before = 0, cost = span.cost(P.C.heads);
    if (chunks > 1) {
        for (uint32_t c = warp; c < chunks; c += S::kWarps) {
            unsigned long long sum = stream_span<S::kCols>(P, 32 * c + lane).cost(P.C.heads);
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
    const unsigned long long runs = (unsigned long long)gridDim.x * S::kWarps, run = (unsigned long long)blockIdx.x * S::kWarps + warp;
    const unsigned long long from = total * run / runs, to = total * (run + 1) / runs;
    const unsigned long long block_from = total * ((unsigned long long)blockIdx.x * S::kWarps) / runs, block_to = total * ((unsigned long long)(blockIdx.x + 1) * S::kWarps) / runs;

    // ---- the place of step `from`: sequence, item of the sequence, step of the item ----
    uint32_t b = 0, item = 0, step = 0;
    unsigned long long item_from = 0;                     // the present item's first step among all
    if (from < to) {
        uint32_t c = 0;
        if (chunks > 1) {
            while (before + s_cost[c] <= from) before += s_cost[c++];
            span = stream_span<S::kCols>(P, 32 * c + lane);
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
        item = (uint32_t)(inside / steps);
        step = (uint32_t)(inside % steps);
        item_from = from - step;
    }

    // ---- copies: one cursor runs ahead ----
    const Waiter wait{P.spin_limit, &s_failed};
    Cursor<S::kCols> ahead;
    ahead.set(span, b, item, step);
    SeqSpan at_span = span;                              // `ahead` may come to the next 32 sequences before
    uint32_t place_base = 0xFFFFFFFFu, place_seq = 0xFFFFFFFFu;
    int pages = 0;
    uint32_t missing = 0;                                 // two bits a stage: its tokens 0..15 and 16..31 have no page
    const unsigned long long count = to - from;
    unsigned long long sent = 0;
    auto send = [&](uint32_t st) {
        // the pages of the next 32 places are kept in the lanes
        const uint32_t t0 = ahead.token(), place = t0 >> P.C.page_shift;
        if (place - place_base >= 32 || place_seq != ahead.b) {
            place_base = place & ~31u;
            place_seq = ahead.b;
            const uint32_t mine = place_base + lane;
            pages = mine < P.B.max_pages && (mine << P.C.page_shift) < (uint32_t)ahead.to && ((mine + 1) << P.C.page_shift) > (uint32_t)ahead.from ? kv_page(P.C, P.B, ahead.b, mine) : -1;
        }
        const uint32_t half = P.C.page_shift == 4;         // pages of 16 tokens: two a step
        const int page0 = __shfl_sync(kAll, pages, place & 31), page1 = __shfl_sync(kAll, pages, (place + half) & 31);
        const bool go0 = page0 >= 0, go1 = half ? page1 >= 0 && place + 1 - place_base < 32 : go0;
        missing = (missing & ~(3u << (2 * st))) | ((go0 ? 0u : 1u) | (go1 ? 0u : 2u)) << (2 * st);
        const uint32_t bytes = ((go0 ? 16u : 0u) + (go1 ? 16u : 0u)) * 2 * (S::kRow + S::kBlocks);
        if (elect_one()) {
            const uint32_t bar = bars + 8 * st, head = ahead.head;
            bar_expect(bar, bytes);
            const uint32_t to_keys = ring + st * S::kStage, to_scales = ring_scales + st * 2 * S::kScales;
            auto part = [&](int page, uint32_t at, uint32_t tokens) {
                const uint32_t row = (((uint32_t)page * P.C.heads + head) << P.C.page_shift) + ((t0 + at) & ((1u << P.C.page_shift) - 1));
                tensor_copy<1>(to_keys + at * S::kRow, &key_map, 0, (int)row, bar);
                tensor_copy<1>(to_keys + S::kTile + at * S::kRow, &value_map, 0, (int)row, bar);
                bulk_copy(to_scales + at * S::kBlocks, P.C.scales[0] + (uint64_t)row * S::kBlocks, tokens * S::kBlocks, bar);
                bulk_copy(to_scales + S::kScales + at * S::kBlocks, P.C.scales[1] + (uint64_t)row * S::kBlocks, tokens * S::kBlocks, bar);
            };
            if (!P.skip_copy) {
                if (half) {
                    if (go0) part(page0, 0, 16);
                    if (go1) part(page1, 16, 16);
                } else if (go0) part(page0, 0, 32);
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
    Cursor<S::kCols> at;
    at.set(at_span, b, item, step);
    float acc[S::kNt][S::kTiles][4], top[S::kNt][2], sum[S::kNt][2], factor[S::kNt][2];
    uint32_t q[S::kNt][S::kDim / 8];
    int lo[S::kNt][2], hi[S::kNt][2], lo_most = 0, hi_least = 0;
    uint32_t ref = 0;
    bool fresh = true, ok = true;
    uint32_t st = 0, parity = 0;
    for (unsigned long long done = 0; done < count; ++done) {
        if (fresh) {
            // the item's columns: queries, limits
            fresh = false;
            ref = 0;
            lo_most = 0;
            hi_least = 0x7FFFFFFF;
#pragma unroll
            for (uint32_t t = 0; t < S::kNt; ++t) {
                float own;
                load_queries<S>(P, at, at.tile * S::kCols + 8 * t + g, i, q[t], own);
                factor[t][0] = __shfl_sync(kAll, own, 8 * i);
                factor[t][1] = __shfl_sync(kAll, own, 8 * i + 4);
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
            lo_most = __reduce_max_sync(kAll, lo_most);
            hi_least = __reduce_min_sync(kAll, hi_least);
        }
        if (!wait.warp(bars + 8 * st, parity)) { ok = false; break; }
        const uint32_t keys = ring + st * S::kStage, values = keys + S::kTile, scales = ring_scales + st * 2 * S::kScales;
        const int t0 = (int)at.token();
        const uint32_t gone = (missing >> (2 * st)) & 3;
        const bool plain = t0 >= lo_most && t0 + (int)kStepTokens <= hi_least && gone == 0;

        // scales: a lane has a token
        uint32_t ks, vs;
        if (S::kBlocks == 4) { ks = lds32(scales + 4 * lane); vs = lds32(scales + S::kScales + 4 * lane); }
        else { ks = lds16(scales + 2 * lane); vs = lds16(scales + S::kScales + 2 * lane); }
        bool hidden = false;
        uint32_t poisoned = 0;                           // tokens with NaN in their values that not every column sees
        if (!plain) {
            const int t = t0 + (int)lane;
            hidden = t < at.from || t >= at.to || (gone >> (lane >> 4)) & 1;
            bool nan = false;
#pragma unroll
            for (uint32_t k = 0; k < S::kBlocks; ++k) nan |= ((vs >> (8 * k)) & 0xFF) == 255;
            if (!S::kFp4) {
#pragma unroll
                for (uint32_t c = 0; c < S::kChunks; ++c) {
                    const uint4 w = lds128(values + swizzled<S::kRow>(lane, c));
                    nan |= nan_bytes(w.x) || nan_bytes(w.y) || nan_bytes(w.z) || nan_bytes(w.w);
                }
            }
            nan = nan && !hidden && !(t >= lo_most && t < hi_least);
            poisoned = __ballot_sync(kAll, nan);
            hidden |= nan;
            if (!S::kFp4 && hidden) {
                const uint32_t zero[4] = {};
#pragma unroll
                for (uint32_t c = 0; c < S::kChunks; ++c) sts128(values + swizzled<S::kRow>(lane, c), zero);
                fence_async_shared();                    // the next copy comes here
            }
        }
        {
            // keys: FP32 factors
            float f[4];
#pragma unroll
            for (uint32_t k = 0; k < S::kBlocks; ++k) f[k] = e8m0_value((ks >> (8 * k)) & 0xFF);
            if (S::kBlocks == 4) sts_f4(key_factors + 16 * lane, f);
            else sts_f2(key_factors + 8 * lane, f);
            // values: over the largest scale so far
            uint32_t s[S::kBlocks], most = 0;
#pragma unroll
            for (uint32_t k = 0; k < S::kBlocks; ++k) {
                s[k] = (vs >> (8 * k)) & 0xFF;
                if (s[k] != 255) most = max(most, s[k]);
            }
            most = __reduce_max_sync(kAll, hidden ? 0u : most);
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
            // [token / 2][block] pairs of two tokens
#pragma unroll
            for (uint32_t k = 0; k < S::kBlocks; ++k)
                sts16(value_factors + ((lane >> 1) * S::kBlocks + k) * 4 + (lane & 1) * 2, hidden ? 0u : value_factor(s[k], ref, S::kLift));
            __syncwarp();
        }

        // logits of 32 tokens: p[t][m][..], m 16 tokens, rows g and g + 8, columns 2i and 2i + 1
        float p[S::kNt][2][4];
#pragma unroll
        for (uint32_t m = 0; m < 2; ++m) {
            float f[2][4];
            const uint32_t row = 16 * m + g;
            if (S::kBlocks == 4) { lds_f4(key_factors + 16 * row, f[0]); lds_f4(key_factors + 16 * (row + 8), f[1]); }
            else { lds_f2(key_factors + 8 * row, f[0]); lds_f2(key_factors + 8 * (row + 8), f[1]); }
#pragma unroll
            for (uint32_t t = 0; t < S::kNt; ++t)
#pragma unroll
                for (int k = 0; k < 4; ++k) p[t][m][k] = 0.0f;
#pragma unroll
            for (uint32_t c = 0; c < S::kChunks; c += 2) {
                uint32_t w[4];
                ldmatrix4(keys + swizzled<S::kRow>(16 * m + (lane & 7) + 8 * ((lane >> 3) & 1), c + (lane >> 4)), w);
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
                        float d[4] = {};
                        mma_f16(d, a[0], a[1], a[2], a[3], q[t][4 * block], q[t][4 * block + 1]);
                        mma_f16(d, a[4], a[5], a[6], a[7], q[t][4 * block + 2], q[t][4 * block + 3]);
                        p[t][m][0] = fmaf(d[0], f[0][block], p[t][m][0]);
                        p[t][m][1] = fmaf(d[1], f[0][block], p[t][m][1]);
                        p[t][m][2] = fmaf(d[2], f[1][block], p[t][m][2]);
                        p[t][m][3] = fmaf(d[3], f[1][block], p[t][m][3]);
                    }
                }
            }
        }

        // weights
        bool grew = false;
        float shrink[S::kNt][2];
#pragma unroll
        for (uint32_t t = 0; t < S::kNt; ++t) {
#pragma unroll
            for (uint32_t m = 0; m < 2; ++m)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    p[t][m][k] *= factor[t][k & 1];
                    if (!plain) {
                        const uint32_t r = 16 * m + g + 8 * (k >> 1);
                        const int tok = t0 + (int)r;
                        const bool seen = tok >= lo[t][k & 1] && tok < hi[t][k & 1] && !((gone >> m) & 1);
                        if (!seen) p[t][m][k] = -INFINITY;
                        else if ((poisoned >> r) & 1) p[t][m][k] = __int_as_float(0x7FFFFFFF);
                    }
                }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float best = fmaxf(fmaxf(p[t][0][k], p[t][0][k + 2]), fmaxf(p[t][1][k], p[t][1][k + 2]));
                best = fmaxf(best, __shfl_xor_sync(kAll, best, 4));
                best = fmaxf(best, __shfl_xor_sync(kAll, best, 8));
                best = fmaxf(best, __shfl_xor_sync(kAll, best, 16));
                grew |= best > top[t][k];
                best = fmaxf(best, top[t][k]);
                shrink[t][k] = best == -INFINITY ? 1.0f : exp2_fast(top[t][k] - best);
                top[t][k] = best;
                const float off = best == -INFINITY ? 0.0f : best - 15.0f;
#pragma unroll
                for (uint32_t m = 0; m < 2; ++m) {
                    p[t][m][k] = exp2_fast(p[t][m][k] - off);
                    p[t][m][k + 2] = exp2_fast(p[t][m][k + 2] - off);
                }
                sum[t][k] = sum[t][k] * shrink[t][k] + ((p[t][0][k] + p[t][0][k + 2]) + (p[t][1][k] + p[t][1][k + 2]));
            }
        }
        if (__any_sync(kAll, grew)) {
#pragma unroll
            for (uint32_t t = 0; t < S::kNt; ++t)
#pragma unroll
                for (uint32_t m = 0; m < S::kTiles; ++m)
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[t][m][k] *= shrink[t][k & 1];
        }

        // weighted values, 16 tokens at a time
#pragma unroll
        for (uint32_t m = 0; m < 2; ++m) {
            uint32_t pb[S::kNt][2];
#pragma unroll
            for (uint32_t t = 0; t < S::kNt; ++t) {
                pb[t][0] = transpose8x8(pack_half(p[t][m][0], p[t][m][1]));
                pb[t][1] = transpose8x8(pack_half(p[t][m][2], p[t][m][3]));
            }
            uint32_t f[2][4];                              // of tokens 2i, 2i + 1 and 2i + 8, 2i + 9
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t where = value_factors + (8 * m + 4 * k + i) * S::kBlocks * 4;
                if (S::kBlocks == 4) { const uint4 v = lds128(where); f[k][0] = v.x; f[k][1] = v.y; f[k][2] = v.z; f[k][3] = v.w; }
                else { lds64(where, f[k][0], f[k][1]); }
            }
#pragma unroll
            for (uint32_t c = 0; c < S::kChunks; c += 2) {
                uint32_t w[4];                             // chunk c, c + 1 of the first eight tokens, then of the next
                ldmatrix4_trans(values + swizzled<S::kRow>(16 * m + 8 * (lane >> 4) + (lane & 7), c + ((lane >> 3) & 1)), w);
#pragma unroll
                for (uint32_t h = 0; h < 2; ++h) {
                    const uint32_t block = S::kFp4 ? c + h : c / 2;
                    constexpr uint32_t kPairs = S::kFp4 ? 4 : 2;
                    uint32_t x[4], y[4];
                    if (S::kFp4) { pairs_fp4(w[h], x); pairs_fp4(w[h + 2], y); }
                    else { pairs_e4m3(w[h], x); pairs_e4m3(w[h + 2], y); }
#pragma unroll
                    for (uint32_t k = 0; k < kPairs; ++k) { x[k] = mul_half2(x[k], f[0][block]); y[k] = mul_half2(y[k], f[1][block]); }
#pragma unroll
                    for (uint32_t u = 0; u < kPairs / 2; ++u)
#pragma unroll
                        for (uint32_t t = 0; t < S::kNt; ++t)
                            mma_f16(acc[t][(c + h) * (kPairs / 2) + u], x[2 * u], x[2 * u + 1], y[2 * u], y[2 * u + 1], pb[t][0], pb[t][1]);
                }
            }
        }
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
            constexpr float kDown = 1.0f / (float)(1u << (S::kLift)) / 32768.0f;       // the weights' 2^15 goes here, once
            const uint32_t slot = item_from < from ? 0u : 1u;            // a run's first part is of an item that began before it
            const uint32_t where = slot == 0 ? first_part : ring;
#pragma unroll
            for (uint32_t t = 0; t < S::kNt; ++t) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t in_tile = 8 * t + 2 * i + k, col = at.tile * S::kCols + in_tile;
                    const float total_weight = sum[t][k] * (1.0f / 32768.0f);
                    const float norm = whole ? (total_weight == 0.0f ? 0.0f : 1.0f / total_weight) : 1.0f;
                    uint8_t* out = nullptr;
                    if (whole && at.has(P, col)) {
                        out = at.out(P, col);
                        if (P.lse && g == 0) P.lse[at.lse(P, col)] = lse_of(top[t][k], total_weight);
                    }
#pragma unroll
                    for (uint32_t m = 0; m < S::kTiles; m += S::kFp4 ? 2 : 1) {
                        constexpr uint32_t kOwn = S::kFp4 ? 4 : 2;         // neighbours of the head's width
                        float v[4];
                        v[0] = acc[t][m][k] * kDown * unit * norm;
                        v[1] = acc[t][m][k + 2] * kDown * unit * norm;
                        if (S::kFp4) {
                            v[2] = acc[t][m + 1][k] * kDown * unit * norm;
                            v[3] = acc[t][m + 1][k + 2] * kDown * unit * norm;
                        }
                        const uint32_t d = 16 * m + kOwn * g;
                        if (out) store_out<kOwn>(P, out, d, v);
                        else if (!whole) {
                            if (S::kFp4) sts_f4(where + (in_tile * S::kPartLd + d) * 4, v);
                            else sts_f2(where + (in_tile * S::kPartLd + d) * 4, v);
                        }
                    }
                    if (!whole && g == 0) {
                        sts_f1(where + (S::kCols * S::kPartLd + in_tile) * 4, top[t][k]);
                        sts_f1(where + (S::kCols * S::kPartLd + S::kCols + in_tile) * 4, total_weight);
                    }
                }
            }
            if (!whole && lane == 0) {
                StreamEntry& e = s_entry[2 * warp + slot];
                e.from = item_from;
                e.to = item_to;
                e.b = at.b;
                e.item = at.item;
                e.there = 1;
            }
            item_from = item_to;
            fresh = true;
        }
        at.next(P, at_span);
    }
    if (!ok) {
        // copies under way end, or are waited for as long as anything else, before the block does
        const unsigned long long open = sent;
        for (uint32_t s = 0; s < S::kStages; ++s)
            if (open > s) settled(bars + 8 * s, (uint32_t)((open - 1 - s) / S::kStages) & 1, P.spin_limit);
        if (lane == 0) atomicOr(P.B.marks, kKvGaveUp);
    }
    __syncthreads();
    BlockEnd* ends = reinterpret_cast<BlockEnd*>(P.workspace) + blockIdx.x;
    if (s_failed) {
        if (threadIdx.x == 0) ends->there = 0;
        return;
    }

    // ---- the block's parts, in order ----
    bool goes_on = false;
    for (uint32_t e = 0; e < 2 * S::kWarps;) {
        if (!s_entry[e].there) { ++e; continue; }
        const StreamEntry one = s_entry[e];
        uint32_t end = e + 1;
        while (end < 2 * S::kWarps && (!s_entry[end].there || s_entry[end].from == one.from)) ++end;
        const bool whole = one.from >= block_from && one.to <= block_to, begins = one.from >= block_from;
        Cursor<S::kCols> c;
        c.set_item(P, one.b, one.item);
        for (uint32_t k = threadIdx.x; k < S::kCols * S::kDim / 4; k += S::kWarps * 32) {
            const uint32_t in_tile = k / (S::kDim / 4), d = k % (S::kDim / 4) * 4, col = c.tile * S::kCols + in_tile;
            float best = -INFINITY;
            for (uint32_t j = e; j < end; ++j)
                if (s_entry[j].there) best = fmaxf(best, lds_f1(part_of<S>(base, j) + (S::kCols * S::kPartLd + in_tile) * 4));
            const float off = best == -INFINITY ? 0.0f : best;
            float v[4] = {}, weight = 0.0f;
            for (uint32_t j = e; j < end; ++j) {
                if (!s_entry[j].there) continue;
                const uint32_t part = part_of<S>(base, j);
                const float w = exp2_fast(lds_f1(part + (S::kCols * S::kPartLd + in_tile) * 4) - off);
                float x[4];
                lds_f4(part + (in_tile * S::kPartLd + d) * 4, x);
#pragma unroll
                for (int n = 0; n < 4; ++n) v[n] = fmaf(x[n], w, v[n]);
                weight = fmaf(lds_f1(part + (S::kCols * S::kPartLd + S::kCols + in_tile) * 4), w, weight);
            }
            if (whole) {
                if (c.has(P, col)) finish_column(P, c, col, d, v, best, weight);
            } else {
                float* to_part = partial_of<S>(P, gridDim.x, blockIdx.x, begins ? 1 : 0);
                *reinterpret_cast<float4*>(to_part + in_tile * S::kDim + d) = make_float4(v[0], v[1], v[2], v[3]);
                if (d == 0) {
                    to_part[S::kCols * S::kDim + in_tile] = best;
                    to_part[S::kCols * S::kDim + S::kCols + in_tile] = weight;
                }
            }
        }
        if (!whole && begins) {
            goes_on = true;
            if (threadIdx.x == 0) *ends = BlockEnd{one.to, total, one.b, one.item, 1, 0};
        }
        e = end;
    }
    if (!goes_on && threadIdx.x == 0) ends->there = 0;
}

// The items that go on from one block to the next: a block for each block that an item begins and does not end in.
template <typename S>
__global__ void __launch_bounds__(S::kCols * S::kDim / 4) kv_join_kernel(const AttentionParams P, uint32_t blocks)
{
    grid_wait();
    grid_launch_dependents();
    const BlockEnd end = reinterpret_cast<const BlockEnd*>(P.workspace)[blockIdx.x];
    if (!end.there) return;
    Cursor<S::kCols> c;
    c.set_item(P, end.b, end.item);
    const uint32_t in_tile = threadIdx.x / (S::kDim / 4), d = threadIdx.x % (S::kDim / 4) * 4, col = c.tile * S::kCols + in_tile;
    const unsigned long long runs = (unsigned long long)blocks * S::kWarps;
    // the last block whose steps begin before the item's end
    uint32_t last = blockIdx.x;
    while (last + 1 < blocks && end.total * ((unsigned long long)(last + 1) * S::kWarps) / runs < end.to) ++last;
    float best = -INFINITY, weight = 0.0f, v[4] = {};
    for (uint32_t k = blockIdx.x; k <= last; ++k) {
        if (k > blockIdx.x && end.total * ((unsigned long long)(k + 1) * S::kWarps) / runs == end.total * ((unsigned long long)k * S::kWarps) / runs) continue;     // no steps
        const float* part = partial_of<S>(P, blocks, k, k == blockIdx.x ? 1 : 0);
        const float4 x = *reinterpret_cast<const float4*>(part + in_tile * S::kDim + d);
        const float t = part[S::kCols * S::kDim + in_tile], w = part[S::kCols * S::kDim + S::kCols + in_tile];
        const float next = fmaxf(best, t), off = next == -INFINITY ? 0.0f : next, old = exp2_fast(best - off), now = exp2_fast(t - off);
        best = next;
        v[0] = v[0] * old + x.x * now;
        v[1] = v[1] * old + x.y * now;
        v[2] = v[2] * old + x.z * now;
        v[3] = v[3] * old + x.w * now;
        weight = weight * old + w * now;
    }
    if (c.has(P, col)) finish_column(P, c, col, d, v, best, weight);
}

}  // namespace zc
