// Attention of many rows over a cache: the tensor cores and the exponentials bound it.
//
// Columns of a sequence and a head (rows times the query heads that share it) are cut into tiles of 256, two matrix instructions' rows; a tile
// with a head is an item, a step is 128 tokens of an item.  As in the other kernel all steps in order are cut into equal runs, here one for each block
// (a block an SM), and parts of items are joined by a second kernel.
//
// Roles: twice four warps have a row of a half of the tile a thread (maxima, exponentials, sums, the weights into tensor memory, results); twice four have a token's keys
// or values a thread and write them as FP16 into shared memory, up to two steps ahead; one issues the matrix instructions.  The halves are half a step apart:
// while one is at its softmax the other's products have the tensor cores, and both use what the eight warps have made of the cache.
//   S = Q K^T: both operands in shared memory, 128-byte swizzle, the head's width fastest.  O += P V: P in tensor memory, in S's place; V as it is written,
// the head's width fastest, which for this product is the outer axis.  S and O, FP32, of both halves are all of tensor memory's 512 columns (head_dim 128).
//   Keys and values are element * 2^(s - R + kLift), R the largest scale byte that the item has met, for keys and for values: exact unless a scale is 2^-35 (E4M3:
// 2^-22) of the largest, off by at most 2^-25 / 2^kLift of 2^R then.  Queries as in the other kernel.
//   Weights are 2^(x - u) as in the other kernel, but u moves only where the largest is beyond 2^15.9, to 2^15 again: so the sums in tensor memory are touched only when a row's
// largest weight grows by a factor of 1.8.  Rounded to FP16: off by at most 2^-12 of it down to 2^-29 of the largest, by 2^-40 of the largest below; the sum of weights is FP32.
//   Measured: 2048 rows, 32 heads, behind 32768 tokens in FP4: 1293 us, 877 TFLOP/s; the tensor cores work 43 % of the time, a half's softmax takes some 3000 of a step's 5200 cycles (the
// special function units 1024 of it).  Two blocks an SM with 128 rows each: 1634 us.  16 warps for the softmax, half a row a thread: 1379 us, the four that are
// left for keys and values do not keep up.  A quarter of the exponentials by a polynomial on the FP32 units: 1 % less time.  (One B200.)  No registers are spilled.
#pragma once
#include "zc_kv_stream.cuh"

namespace zc {

template <bool FP4_, uint32_t DIM_>
struct PromptShape {
    static constexpr bool kFp4 = FP4_;
    static constexpr uint32_t kDim = DIM_, kCols = 256, kStep = 128;
    static constexpr uint32_t kRow = kFp4 ? kDim / 2 : kDim, kBlocks = kDim / kKvBlock;
    static constexpr int kLift = kFp4 ? 12 : 6;                              // 6 * 2^12 and 448 * 2^6 are FP16 numbers
    static constexpr uint32_t kTile = 128 * kDim * 2;                        // 128 rows of FP16, pieces of 64 of the head's width one after the other
    static constexpr uint32_t kSmem = 6 * kTile + 1024;                      // queries of both halves; keys and values of two steps
    static constexpr uint32_t kThreads = 17 * 32;
    static constexpr uint32_t kHalf = 256, kO = 128, kTmem = 512;            // columns: of a half S, then O
};

// Where a role is; the same in all of a block's threads.
struct PromptCursor : SeqRows {
    uint32_t b, tile, head, tiles, step, steps, first_step;
    __device__ __forceinline__ void tile_span(const AttentionParams& P, uint32_t t, uint32_t& first, uint32_t& count) const
    {
        const uint32_t cols = (uint32_t)n * P.group, last = min(cols, (t + 1) * 256) - 1;
        int lo, hi, skip;
        limits(P, (int)(last / P.group), skip, hi);
        limits(P, (int)(t * 256 / P.group), lo, skip);
        hi = min(max(hi, 0), len);
        first = (uint32_t)lo / 128;
        const uint32_t end = ((uint32_t)hi + 127) / 128;
        count = end > first ? end - first : 1;             // at least one, that rows which see nothing get their zeros
    }
    __device__ __forceinline__ void sequence(const AttentionParams& P, uint32_t b_)
    {
        b = b_;
        load(P, b);
        tiles = (uint32_t)n > P.most_rows || P.most_rows == 0xFFFFFFFFu ? (uint32_t)(((unsigned long long)n * P.group + 255) / 256) : 0;
    }
    __device__ __forceinline__ void next_item(const AttentionParams& P)
    {
        step = 0;
        if (++head < P.C.heads) return;
        head = 0;
        if (++tile >= tiles) {
            tile = 0;
            do {
                if (b + 1 >= P.B.n_seqs) return;
                sequence(P, b + 1);
            } while (tiles == 0);
        }
        tile_span(P, tile, first_step, steps);
    }
    __device__ __forceinline__ ItemColumns columns(const AttentionParams& P) const { return ItemColumns{row0, head, tile * 256, columns_left(P)}; }
    __device__ __forceinline__ uint32_t columns_left(const AttentionParams& P) const { return min(256u, (uint32_t)n * P.group - tile * 256); }
};

__device__ __forceinline__ void mma_ss_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
__device__ __forceinline__ void mma_ts_f16(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" :: "r"(d), "r"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
// 32 columns of a warp's 32 lanes; not complete before tmem_ld_wait
__device__ __forceinline__ void tmem_ld32_async(uint32_t addr, float v[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
                   "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
                   "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]),
                   "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
                 : "r"(addr));
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t v[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 :: "r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
                    "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const float v[32])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
                 :: "r"(addr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]),
                    "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]),
                    "f"(v[16]), "f"(v[17]), "f"(v[18]), "f"(v[19]), "f"(v[20]), "f"(v[21]), "f"(v[22]), "f"(v[23]),
                    "f"(v[24]), "f"(v[25]), "f"(v[26]), "f"(v[27]), "f"(v[28]), "f"(v[29]), "f"(v[30]), "f"(v[31]) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// A tile whose rows are tokens and whose outer axis for the product is the head's width: pieces of 64 of it 128 rows * 128 bytes apart, groups of 8 rows 1024 bytes.
__device__ __forceinline__ uint64_t outer_desc(uint32_t addr)
{
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(16384 >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// Where 16 bytes (8 of the head's width) of a row of a tile are.
__device__ __forceinline__ uint32_t tile_at(uint32_t row, uint32_t chunk) { return (chunk >> 3) * 16384 + row * 128 + (((chunk ^ row) & 7) << 4); }

// 2^(s - ref + lift) in FP16, twice; NaN for 255.
__device__ __forceinline__ uint32_t element_factor(uint32_t s, uint32_t ref, int lift)
{
    const int e = (int)s - (int)ref + lift + 15;
    return (s == 255 ? 0x7E00u : e > 0 ? (uint32_t)e << 10 : 0x400u >> min(1 - e, 31)) * 0x10001u;
}

// One token's elements, raw in w, into its row of a tile.
template <typename S>
__device__ __forceinline__ void write_row(uint32_t tile, uint32_t row, const uint4* w, uint32_t scales, uint32_t ref, bool hidden)
{
#pragma unroll
    for (uint32_t k = 0; k < S::kBlocks; ++k) {
        const uint32_t f = hidden ? 0u : element_factor((scales >> (8 * k)) & 0xFF, ref, S::kLift);
        if (S::kFp4) {
            const uint32_t x[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                uint32_t h[4];
                fp4_to_half(x[j], h);
#pragma unroll
                for (int i = 0; i < 4; ++i) h[i] = mul_half2(h[i], f);
                sts128(tile + tile_at(row, 4 * k + j), h);
            }
        } else {
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                const uint4 v = w[2 * k + j / 2];
                const uint32_t x0 = j & 1 ? v.z : v.x, x1 = j & 1 ? v.w : v.y;
                uint32_t h[4];
                e4m3_to_half(x0, h);
                e4m3_to_half(x1, h + 2);
#pragma unroll
                for (int i = 0; i < 4; ++i) h[i] = hidden ? 0u : mul_half2(h[i], f);
                sts128(tile + tile_at(row, 4 * k + j), h);
            }
        }
    }
}

// Two numbers at once.
__device__ __forceinline__ void fma_pair(float& x, float& y, float m, float a)
{
    asm("{\n\t.reg .b64 v, w, z;\n\tmov.b64 v, {%0, %1};\n\tmov.b64 w, {%2, %2};\n\tmov.b64 z, {%3, %3};\n\tfma.rn.f32x2 v, v, w, z;\n\tmov.b64 {%0, %1}, v;\n\t}"
        : "+f"(x), "+f"(y) : "f"(m), "f"(a));
}
__device__ __forceinline__ void add_pair(float& x, float& y, float a, float b)
{
    asm("{\n\t.reg .b64 v, w;\n\tmov.b64 v, {%0, %1};\n\tmov.b64 w, {%2, %3};\n\tadd.rn.f32x2 v, v, w;\n\tmov.b64 {%0, %1}, v;\n\t}" : "+f"(x), "+f"(y) : "f"(a), "f"(b));
}
__device__ __forceinline__ void mul_pair(float& x, float& y, float m)
{
    asm("{\n\t.reg .b64 v, w;\n\tmov.b64 v, {%0, %1};\n\tmov.b64 w, {%2, %2};\n\tmul.rn.f32x2 v, v, w;\n\tmov.b64 {%0, %1}, v;\n\t}" : "+f"(x), "+f"(y) : "f"(m));
}

template <typename S>
__global__ void __launch_bounds__(S::kThreads, 1) kv_prompt_kernel(const AttentionParams P)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ __align__(8) uint64_t s_bars[16];
    __shared__ uint32_t s_tmem;
    __shared__ volatile uint32_t s_failed;
    __shared__ unsigned long long s_total, s_item_from;
    __shared__ uint32_t s_start[4];                       // sequence, tile, head, step
    // by step parity:
    __shared__ uint32_t s_most[2][2][4];                  // largest scale bytes of keys and values, by warp
    __shared__ uint32_t s_ref[2][2];                      // what keys and values are over
    __shared__ uint32_t s_gone[2][4], s_poisoned[2][4];   // tokens without a page; with NaN in their values that not every row sees
    constexpr uint32_t kAll = 0xFFFFFFFFu;
    const uint32_t lane = threadIdx.x & 31, warp = warp_index();
    const uint32_t base = (smem_u32(smem) + 1023) & ~1023u, q_tile = base, k_tile = base + 2 * S::kTile, v_tile = base + 4 * S::kTile;
    const uint32_t bars = smem_u32(s_bars);
    // of each half: queries written; first product done; weights written; second product done.  Of each step parity: keys written and values' scales known; values written; both used.  Of keys and values: scales known
    const uint32_t q_full = bars, s_full = bars + 16, p_full = bars + 32, o_full = bars + 48, k_full = bars + 64, v_full = bars + 80, kv_free = bars + 96, m_full = bars + 112;
    if (threadIdx.x == 0) {
        s_failed = 0;
        for (uint32_t x = 0; x < 2; ++x) {
            bar_init(q_full + 8 * x, 128);
            bar_init(s_full + 8 * x, 1);
            bar_init(p_full + 8 * x, 128);
            bar_init(o_full + 8 * x, 1);
            bar_init(k_full + 8 * x, 256);
            bar_init(v_full + 8 * x, 128);
            bar_init(kv_free + 8 * x, 1);
        }
        bar_init(m_full, 4);
        bar_init(m_full + 8, 4);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 16) tmem_alloc<1>(smem_u32(&s_tmem), S::kTmem);
    grid_wait();
    grid_launch_dependents();

    // ---- which steps are this block's: every tile of every sequence is looked at, 32 at a time ----
    if (warp == 0) {
        unsigned long long total = 0;
        for (int pass = 0; pass < 2; ++pass) {
            const uint32_t blocks = working_blocks(total, 1, gridDim.x);
            if (pass && blockIdx.x >= blocks) break;
            const unsigned long long from = pass ? share(total, blockIdx.x, blocks) : 0;
            unsigned long long before = 0;
            bool found = false;
            PromptCursor many{};                          // a lane has one of 32 sequences
            for (uint32_t b = 0; b < P.B.n_seqs && !found; ++b) {
                if ((b & 31) == 0) {
                    many.tiles = 0;
                    if (b + lane < P.B.n_seqs) many.sequence(P, b + lane);
                }
                PromptCursor c;
                c.tiles = __shfl_sync(kAll, many.tiles, b & 31);
                if (c.tiles == 0) continue;
                c.n = __shfl_sync(kAll, many.n, b & 31);
                c.len = __shfl_sync(kAll, many.len, b & 31);
                for (uint32_t t0 = 0; t0 < c.tiles; t0 += 32) {
                    uint32_t first = 0, count = 0;
                    if (t0 + lane < c.tiles) c.tile_span(P, t0 + lane, first, count);
                    unsigned long long upto = (unsigned long long)count * P.C.heads;
                    for (int d = 1; d < 32; d <<= 1) {
                        const unsigned long long o = __shfl_up_sync(kAll, upto, d);
                        if ((int)lane >= d) upto += o;
                    }
                    const unsigned long long sum = __shfl_sync(kAll, upto, 31);
                    if (pass && before + sum > from) {
                        const uint32_t k = __ffs(__ballot_sync(kAll, before + upto > from)) - 1;
                        const uint32_t steps = __shfl_sync(kAll, count, k);
                        const unsigned long long inside = from - before - (__shfl_sync(kAll, upto, k) - (unsigned long long)steps * P.C.heads);
                        if (lane == 0) {
                            uint32_t head = 0;               // below 2^10
                            for (uint32_t bit = ZC_KV_MAX_HEADS / 2; bit; bit /= 2)
                                if ((unsigned long long)(head + bit) * steps <= inside) head += bit;
                            const uint32_t step = (uint32_t)(inside - (unsigned long long)head * steps);
                            s_start[0] = b;
                            s_start[1] = t0 + k;
                            s_start[2] = head;
                            s_start[3] = step;
                            s_item_from = from - step;
                        }
                        found = true;
                        break;
                    }
                    before += sum;
                }
            }
            if (!pass) total = before;
        }
        if (lane == 0) s_total = total;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const unsigned long long total = s_total;
    const uint32_t blocks = working_blocks(total, 1, gridDim.x);
    const unsigned long long from = blockIdx.x < blocks ? share(total, blockIdx.x, blocks) : 0, to = blockIdx.x < blocks ? share(total, blockIdx.x + 1, blocks) : 0;
    const bool endless = (to - from) >> 32 != 0;          // three hours at 2.6 us a step: not begun
    const uint32_t count = endless ? 0u : (uint32_t)(to - from), tmem = __shfl_sync(kAll, s_tmem, 0);
    const KvWaiter wait{P.spin_limit, smem_u32(const_cast<uint32_t*>(&s_failed))};
    if (endless) wait.give_up();
    PromptCursor c;
    if (count) {
        c.sequence(P, s_start[0]);
        c.tile = s_start[1];
        c.head = s_start[2];
        c.step = s_start[3];
        c.tile_span(P, c.tile, c.first_step, c.steps);
    }
    BlockEnd* ends = reinterpret_cast<BlockEnd*>(P.workspace) + blockIdx.x;
    uint32_t first_done[2] = {}, second_done[2] = {};      // of the issuing warp: products issued, of each half

    if (warp == 16) {
        // ---- matrix instructions ----
        const uint32_t qk = (1u << 4) | ((128u >> 3) << 17) | ((128u >> 4) << 24);                               // FP16 operands, FP32 sums
        const uint32_t pv = (1u << 4) | (1u << 16) | ((S::kDim >> 3) << 17) | ((128u >> 4) << 24);               // the second operand by its outer axis
        uint32_t items[2] = {};
        const uint64_t q_desc = operand_desc(q_tile), k_desc = operand_desc(k_tile), v_desc = outer_desc(v_tile);        // addresses in units of 16 bytes
        // a half's first product for step j; `fresh`: of a new item
        auto first = [&](uint32_t x, uint32_t j, bool fresh) -> bool {
            if (fresh && !wait.warp(q_full + 8 * x, items[x]++ & 1)) return false;
            if (!wait.warp(k_full + 8 * (j & 1), (j >> 1) & 1)) return false;
            tc_fence_after();
            if (P.skip_math) { wait.give_up(); return false; }
            const uint64_t q = q_desc + x * (S::kTile >> 4), keys = k_desc + (j & 1) * (S::kTile >> 4);
            if (elect_one()) {
#pragma unroll
                for (uint32_t k = 0; k < S::kDim / 16; ++k) {
                    const uint32_t off = ((k >> 2) * 16384 + (k & 3) * 32) >> 4;
                    mma_ss_f16(tmem + x * S::kHalf, q + off, keys + off, qk, k != 0);
                }
                mma_commit<1>(s_full + 8 * x);
            }
            __syncwarp();
            ++first_done[x];
            return true;
        };
        uint32_t halves = 0;
        bool ok = true, fresh = true;
        if (count) {
            halves = c.columns_left(P) > 128 ? 2 : 1;
            for (uint32_t x = 0; x < halves && ok; ++x) ok = first(x, 0, true);
        }
        for (uint32_t j = 0; j < count && ok; ++j) {
            PromptCursor n = c;
            const bool item_ends = c.step + 1 == c.steps;
            if (item_ends) n.next_item(P);
            else ++n.step;
            const uint32_t next_halves = item_ends && j + 1 < count ? (n.columns_left(P) > 128 ? 2 : 1) : halves;
            for (uint32_t x = 0; x < 2 && ok; ++x) {
                if (x < halves) {
                    if (!wait.warp(v_full + 8 * (j & 1), (j >> 1) & 1) || !wait.warp(p_full + 8 * x, second_done[x] & 1)) { ok = false; break; }
                    tc_fence_after();
                    const uint64_t values = v_desc + (j & 1) * (S::kTile >> 4);
                    if (elect_one()) {
#pragma unroll
                        for (uint32_t k = 0; k < 8; ++k)
                            mma_ts_f16(tmem + x * S::kHalf + S::kO, tmem + x * S::kHalf + 8 * k, values + k * (2048 >> 4), pv, !(fresh && k == 0));
                        mma_commit<1>(o_full + 8 * x);
                        if (x + 1 == halves) mma_commit<1>(kv_free + 8 * (j & 1));
                    }
                    __syncwarp();
                    ++second_done[x];
                }
                if (j + 1 < count && x < next_halves) {
                    // the product goes where the last step's weights are
                    if (second_done[x] && !wait.warp(o_full + 8 * x, (second_done[x] - 1) & 1)) { ok = false; break; }
                    ok = first(x, j + 1, item_ends);
                }
            }
            halves = next_halves;
            fresh = item_ends;
            c = n;
        }
    } else if (warp >= 8) {
        // ---- keys (side 0) and values (side 1): a thread has a token ----
        const uint32_t row = threadIdx.x & 127, group = row >> 5, side = (warp >> 2) & 1;
        PromptCursor ahead = c;                            // the step whose elements are read, one ahead
        constexpr uint32_t kWords = S::kRow / 16;
        uint4 now[kWords], next[kWords];
        uint32_t now_scales = 0, next_scales = 0;
        int now_page = -2, next_page = -2, later_page = -2;
        auto find_page = [&](const PromptCursor& a) -> int {
            const uint32_t t = (a.first_step + a.step) * 128 + row;
            int lo, hi, skip;
            a.limits(P, (int)(a.tile * 256 / P.group), lo, skip);
            a.limits(P, (int)((a.tile * 256 + a.columns_left(P) - 1) / P.group), skip, hi);
            return (int)t >= lo && (int)t < hi && t < (uint32_t)a.len ? kv_page(P.C, P.B, a.b, t >> P.C.page_shift) : -2;     // -2: nobody sees the token
        };
        const uint8_t *elems = P.C.elems[side], *scales = P.C.scales[side];
        auto load = [&](const PromptCursor& a, int pg) {
            const uint32_t t = (a.first_step + a.step) * 128 + row;
            if (pg >= 0) {
                const uint64_t at = (((uint64_t)pg * P.C.heads + a.head) << P.C.page_shift) + (t & ((1u << P.C.page_shift) - 1));
                const uint4* w = reinterpret_cast<const uint4*>(elems + at * S::kRow);
#pragma unroll
                for (uint32_t i = 0; i < kWords; ++i) next[i] = w[i];
                next_scales = S::kBlocks == 4 ? *reinterpret_cast<const uint32_t*>(scales + at * 4) : *reinterpret_cast<const uint16_t*>(scales + at * 2);
            }
        };
        auto advance = [&](PromptCursor& a) { if (++a.step == a.steps) a.next_item(P); };
        uint32_t ref = 0;
        const uint32_t tile = side ? v_tile : k_tile, full = side ? v_full : k_full, known = m_full + 8 * side;
        if (count) {
            next_page = find_page(ahead);
            load(ahead, next_page);
            advance(ahead);
            if (count > 1) later_page = find_page(ahead);
        }
        for (uint32_t j = 0; j < count; ++j) {
            const uint32_t par = j & 1;
            // the next step's elements are on their way while this one's are written, its pages a step earlier
#pragma unroll
            for (uint32_t i = 0; i < kWords; ++i) now[i] = next[i];
            now_scales = next_scales;
            now_page = next_page;
            next_page = later_page;
            if (j + 1 < count) {
                load(ahead, next_page);
                if (j + 2 < count) {
                    advance(ahead);
                    later_page = find_page(ahead);
                }
            }
            // the step before the last is over: its keys, values, and what is said of them
            if (j >= 2 && !wait.warp(kv_free + 8 * par, ((j >> 1) - 1) & 1)) break;
            if (j && c.step == 0) ref = 0;
            const bool hidden = now_page < 0;
            // the largest scales
            uint32_t most = 0;
            bool nan = false;
            if (!hidden) {
#pragma unroll
                for (uint32_t k = 0; k < S::kBlocks; ++k) {
                    const uint32_t a = (now_scales >> (8 * k)) & 0xFF;
                    if (a != 255) most = max(most, a);
                    nan |= a == 255;
                }
                if (!S::kFp4 && side) {
#pragma unroll
                    for (uint32_t i = 0; i < kWords; ++i) nan |= nan_bytes(now[i].x) || nan_bytes(now[i].y) || nan_bytes(now[i].z) || nan_bytes(now[i].w);
                }
            }
            nan = nan && side;
            if (nan) {
                // NaN in values that every row of the tile sees goes through the product, else the rows that see it are told
                const int t = (int)((c.first_step + c.step) * 128 + row);
                int lo, hi, skip;
                c.limits(P, (int)(c.tile * 256 / P.group), skip, hi);
                c.limits(P, (int)((c.tile * 256 + c.columns_left(P) - 1) / P.group), lo, skip);
                nan = t < lo || t >= hi;
            }
            most = __reduce_max_sync(kAll, most);
            const uint32_t gone = __ballot_sync(kAll, now_page == -1), poisoned = __ballot_sync(kAll, nan);
            if (lane == 0) {
                s_most[par][side][group] = most;
                if (side) s_poisoned[par][group] = poisoned;
                else s_gone[par][group] = gone;
                bar_arrive(known);
            }
            if (!wait.warp(known, par)) break;
#pragma unroll
            for (int k = 0; k < 4; ++k) ref = max(ref, s_most[par][side][k]);
            if (row == 0) s_ref[par][side] = ref;
            if (side) bar_arrive(k_full + 8 * par);        // what is said of the values comes with the keys
            write_row<S>(tile + par * S::kTile, row, now, now_scales, ref, hidden || nan);
            fence_async_shared();
            bar_arrive(full + 8 * par);
            advance(c);
        }
    } else {
        // ---- rows of a half: a thread has one ----
        const uint32_t half = warp >> 2, row = threadIdx.x & 127, at = tmem + half * S::kHalf + (((warp & 3) * 32) << 16);
        const uint32_t my_s = s_full + 8 * half, my_p = p_full + 8 * half, my_o = o_full + 8 * half;
        unsigned long long item_from = s_item_from;
        float top = -INFINITY, sum = 0.0f;
        int lo = 0, hi = 0x7FFFFFFF, lo_most = 0, hi_least = 0;
        uint32_t col = 0, v_ref = 0, turns = 0;               // turns: steps in which the half had rows
        uint32_t idle = 0;                                    // steps since then in which it had none
        int up = 0;                                           // the query is over 2^-up
        bool fresh = true, goes_on = false;
        for (uint32_t j = 0; j < count; ++j) {
            const uint32_t par = j & 1, cols = (uint32_t)c.n * P.group, first_col = c.tile * 256 + half * 128;
            const bool item_ends = c.step + 1 == c.steps, active = first_col < cols;
            if (active) {
                if (fresh) {
                    col = first_col + row;
                    int skip;
                    lo = 0;
                    hi = 0x7FFFFFFF;
                    if (col < cols) c.limits(P, (int)(col / P.group), lo, hi);
                    c.limits(P, (int)((min(cols, first_col + 128) - 1) / P.group), lo_most, skip);
                    c.limits(P, (int)(first_col / P.group), skip, hi_least);
                    hi_least = min(hi_least, c.len);
                    // the query over a power of two, in FP16; twice read, the second time out of the L1; eight reads under way at a time
                    const uint8_t* q = P.q.d + (uint64_t)(c.row0 + col / P.group) * P.q.ld_row + (uint64_t)(c.head * P.group + col % P.group) * P.q.ld_head;
                    float most = 0.0f;
                    if (col < cols)
                        for (uint32_t k = 0; k < S::kDim / 4; k += 8) {
                            uint2 w[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) w[i] = query_four(P, q + 8 * (k + i));
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const float2 x = query_pair(P, w[i].x), y = query_pair(P, w[i].y);
                                most = fmaxf(fmaxf(most, fmaxf(fabsf(x.x), fabsf(x.y))), fmaxf(fabsf(y.x), fabsf(y.y)));
                            }
                        }
                    up = query_lift(most);
                    const float lift = copysignf(power_of_two(up), P.scale_mantissa);
                    for (uint32_t k = 0; k < S::kDim / 8; k += 4) {
                        uint2 w[8] = {};
                        if (col < cols)
#pragma unroll
                            for (int i = 0; i < 8; ++i) w[i] = query_four(P, q + 16 * k + 8 * i);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint32_t h[4];
#pragma unroll
                            for (int n = 0; n < 4; ++n) {
                                const float2 x = query_pair(P, n & 1 ? w[2 * i + n / 2].y : w[2 * i + n / 2].x);
                                h[n] = pack_half(x.x * lift, x.y * lift);
                            }
                            sts128(q_tile + half * S::kTile + tile_at(row, k + i), h);
                        }
                    }
                    fence_async_shared();
                    bar_arrive(q_full + 8 * half);
                    top = -INFINITY;
                    sum = 0.0f;
                }
                // the limit is a step's: a half that had no rows for some steps is that many ahead of the others
                if (!KvWaiter{(uint32_t)min((unsigned long long)wait.limit * (idle + 1), 0xFFFFFFFEull), wait.failed}.warp(my_s, turns & 1)) break;
                idle = 0;
                tc_fence_after();
                const int t0 = (int)((c.first_step + c.step) * 128);
                const uint32_t k_ref = s_ref[par][0], new_ref = s_ref[par][1];
                const bool plain = t0 >= lo_most && t0 + 128 <= hi_least && (s_gone[par][0] | s_gone[par][1] | s_gone[par][2] | s_gone[par][3]) == 0 &&
                                   (s_poisoned[par][0] | s_poisoned[par][1] | s_poisoned[par][2] | s_poisoned[par][3]) == 0;
                float f = logit_factor(P, (int)k_ref - 127 - S::kLift - up);
                if (!plain) {
                    // what the row does not see, in place
#pragma unroll 1
                    for (uint32_t k = 0; k < 4; ++k) {
                        const uint32_t gone = s_gone[par][k], poisoned = s_poisoned[par][k];
                        float v[32];
                        tmem_ld32_async(at + 32 * k, v);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            const int t = t0 + (int)(32 * k) + i;
                            if ((poisoned >> i) & 1) v[i] = __int_as_float(0x7FFFFFFF);
                            if (t < lo || t >= hi || t >= c.len || ((gone >> i) & 1)) v[i] = -INFINITY;
                        }
                        tmem_st32(at + 32 * k, v);
                    }
                    tmem_st_wait();
                }
                float most[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
                for (uint32_t k = 0; k < 4; ++k) {
                    float v[32];
                    tmem_ld32_async(at + 32 * k, v);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 16; ++i) most[i & 3] = fmaxf(most[i & 3], fmaxf(v[2 * i], v[2 * i + 1]));
                }
                const float best = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])) * f;
                // the sums in tensor memory are over 2^top of the weights and 2^v_ref of the values
                float shrink = move_unit(top, best, 15.9f);
                sum *= shrink;
                if (!fresh && new_ref != v_ref) shrink *= ldexpf(1.0f, max((int)v_ref - (int)new_ref, -200));
                if (__any_sync(kAll, shrink != 1.0f || fabsf(best) >= kFarLogit)) {
                    if (!fresh) {
#pragma unroll 1
                        for (uint32_t k = 0; k < S::kDim / 32; ++k) {
                            float v[32];
                            tmem_ld32_async(at + S::kO + 32 * k, v);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 32; i += 2) mul_pair(v[i], v[i + 1], shrink);
                            tmem_st32(at + S::kO + 32 * k, v);
                        }
                    }
                    if (__any_sync(kAll, fabsf(best) >= kFarLogit && best != -INFINITY)) {
                        // logits as large as this are rounded before their differences are taken
#pragma unroll 1
                        for (uint32_t k = 0; k < 4; ++k) {
                            float v[32];
                            tmem_ld32_async(at + 32 * k, v);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 32; i += 2) mul_pair(v[i], v[i + 1], f);
                            tmem_st32(at + 32 * k, v);
                        }
                        tmem_st_wait();
                        f = 1.0f;
                    }
                }
                v_ref = new_ref;
                const float off = top == -INFINITY ? 0.0f : -top;
                float more[2] = {0.0f, 0.0f};
#pragma unroll 1
                for (uint32_t k = 0; k < 4; ++k) {
                    float v[32];
                    uint32_t h[16];
                    tmem_ld32_async(at + 32 * k, v);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        fma_pair(v[2 * i], v[2 * i + 1], f, off);
                        v[2 * i] = exp2_fast(v[2 * i]);
                        v[2 * i + 1] = exp2_fast(v[2 * i + 1]);
                        add_pair(more[0], more[1], v[2 * i], v[2 * i + 1]);
                        h[i] = pack_half(v[2 * i], v[2 * i + 1]);
                    }
                    tmem_st16(at + 16 * k, h);
                }
                sum += more[0] + more[1];
                tmem_st_wait();
                tc_fence_before();
                bar_arrive(my_p);
                if (item_ends || j + 1 == count) {
                    if (!wait.warp(my_o, turns & 1)) break;
                    tc_fence_after();
                    const unsigned long long item_to = item_from + c.steps;
                    const bool begins = item_from >= from, whole = begins && item_to <= to;
                    const float weight = sum;
                    constexpr float kDown = 1.0f / (float)(1u << S::kLift);
                    const float unit = e8m0_value(v_ref), norm = kDown * inverse_weight(weight);        // before `unit`: the sum itself may be beyond FP32
                    const bool mine = col < cols;
                    const uint32_t head = c.head * P.group + col % P.group;
                    const uint64_t out_row = (uint64_t)c.row0 + col / P.group;
                    uint8_t* out = P.out.d + out_row * P.out.ld_row + head * P.out.ld_head;
                    float* part = partial_of<S>(P, gridDim.x, blockIdx.x, begins ? 1 : 0);
#pragma unroll 1
                    for (uint32_t k = 0; k < S::kDim / 32; ++k) {
                        float v[32];
                        tmem_ld32_async(at + S::kO + 32 * k, v);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = v[i] * norm * unit;
                        if (!mine) continue;
#pragma unroll
                        for (int i = 0; i < 32; i += 4) {
                            if (whole) store_out<4>(P, out, 32 * k + i, v + i);
                            else *reinterpret_cast<float4*>(part + (half * 128 + row) * S::kDim + 32 * k + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                        }
                    }
                    if (mine && whole && P.lse) P.lse[out_row * P.q_heads + head] = lse_of(top, weight);
                    if (!whole) {
                        part[S::kCols * S::kDim + half * 128 + row] = top;
                        part[S::kCols * S::kDim + S::kCols + half * 128 + row] = weight;
                        if (begins) {
                            goes_on = true;
                            if (threadIdx.x == 0) *ends = BlockEnd{item_to, total, c.columns(P), 1, {}};
                        }
                    }
                    tc_fence_before();                     // read before the next item's products
                }
                ++turns;
            } else ++idle;
            fresh = item_ends;
            if (item_ends) {
                item_from += c.steps;
                c.next_item(P);
            } else ++c.step;
        }
        if (threadIdx.x == 0 && !goes_on) ends->there = 0;
    }
    __syncthreads();
    if (warp == 16) {
        // products under way end, or are waited for as long as anything else, before the block and its memories are given back
        if (s_failed) {
            for (uint32_t x = 0; x < 2; ++x) {
                if (first_done[x]) settled(s_full + 8 * x, (first_done[x] - 1) & 1, P.spin_limit);
                if (second_done[x]) settled(o_full + 8 * x, (second_done[x] - 1) & 1, P.spin_limit);
            }
            if (lane == 0) {
                atomicOr(P.B.marks, kKvGaveUp);
                ends->there = 0;
            }
        }
        tc_fence_after();
        tmem_free<1>(tmem, S::kTmem);
    }
}

}  // namespace zc
