// zc_fp8_moe: a mixture-of-experts layer for a few tokens, in two kernels.
//
// With a few tokens the time goes into reading the chosen experts' weights once.  They are streamed by tensor copies into shared
// memory and multiplied there as they are, FP8 with their scale bytes, on the fifth-generation tensor cores: no thread ever
// touches a weight.  (Widening them in registers for warp-wide BF16 instructions took 350 instructions per KiB and ran at a
// sixth of the memory's rate.)  The instruction wants FP8 on the other side as well, so an activation is written as a sum of
// E4M3 pieces, v = 2^s (q0 + 2^-4 q1 + 2^-8 q2 + ...), with s from the largest magnitude of 128 columns: q_i is what the
// pieces before it leave, rounded.  The first leaves 2^-4 of the value, every other one, with four bits and a sign for what is at
// most half a step, 2^-5 of that.  Three pieces hold BF16 and FP16 exactly (8 and 11 bits) down to 2^-17 of the largest of
// the 128, and nothing smaller is off by more than 2^-25 of it.  The pieces are rows of the same operand, so they cost columns of
// the accumulator, and their sum is taken in FP32 at the end.
//
// Rows are handed out in groups of eight, the swizzle's height, in tiles whose height is chosen so that the blocks get equal numbers
// of them (cut_rows); the tiles of all chosen experts form one sequence, of which each block takes a stretch.
//
//   kernel 1  routes (every cluster for itself, so that no block waits for another cluster), then gate and up: a tile is up to 64
//             rows of gate and the same rows of up; the result warps of the two give each other half of the tokens
//   kernel 2  down: up to 128 rows a tile, one FP32 row of partial results per (token, expert); the block that completes a
//             group's last expert adds the experts up in the order of the token's list, when it has done all its tiles
//
// Warps of a block: 0 tensor copies, 1 matrix instructions, 2 the weights' scale bytes, 4-7 results, 8-23 the activations' pieces.
#include "zc_fp8_tensor.cuh"

namespace zc {

constexpr uint32_t kMoeWarps = 24, kMoeThreads = 32 * kMoeWarps;
constexpr uint32_t kMoeCluster = 4;
constexpr uint32_t kMaxTokens = ZC_FP8_MOE_MAX_TOKENS, kMaxExperts = ZC_FP8_MOE_MAX_EXPERTS;
constexpr uint32_t kMaxRows = kMaxTokens * ZC_FP8_MOE_MAX_TOP_K;
constexpr uint32_t kBuilders = 16;               // warps that make pieces
constexpr uint32_t kMoeMaxStages = 9;
constexpr uint32_t kMoeStageSpace = 208896;      // shared memory for stages: weights, pieces, 1 KiB of scale words each
// Steps of down (2048 columns) after which the accumulator, which cuts off what does not fit every 32 columns, is added to the partial
// result in FP32, to nearest: sums of one sign over 14336 columns are less than 6e-6 short, 1.3e-5 in one accumulator; y of experts 14336
// wide is 5e-5 to 9e-5 from an FP32 form's (norm), 8e-5 to 1.4e-4 in one accumulator; in the same time.
constexpr uint32_t kPartSteps = 16;
constexpr uint32_t kMoeHeights = 5;              // tensor copies of 8, 16, 32, 64 and 128 rows
// Tiles that complete a band at most: a block has up to 4 tiles per pass of an expert (8192 groups of rows in tiles of 16 on more than
// 128 blocks) and 31 more, so it touches fewer bands than this; launch_moe refuses a GPU with so few SMs that it would not.
constexpr uint32_t kMoeTodo = 64;
constexpr uint32_t kMoeTmemCols = 512;           // two accumulators of 128 columns, then 4 + 4 scale columns per stage
constexpr uint32_t kMoeTmemScales = 256;

struct MoeMaps { CUtensorMap of[kMoeHeights]; };

// rows of pieces of `count` tokens: each piece's rounded up to 8, all to 16 (what is behind the last piece is multiplied and not used)
__host__ __device__ constexpr uint32_t piece_rows(uint32_t count, uint32_t pieces) { return (((count + 7) & ~7u) * pieces + 15) & ~15u; }
__host__ __device__ constexpr uint32_t stage_size(uint32_t pass, uint32_t pieces) { return 16384 + piece_rows(pass, pieces) * 128 + 1024; }
__host__ __device__ constexpr uint32_t stage_count(uint32_t pass, uint32_t pieces)
{
    return kMoeStageSpace / stage_size(pass, pieces) < kMoeMaxStages ? kMoeStageSpace / stage_size(pass, pieces) : kMoeMaxStages;
}
static_assert(piece_rows(16, 4) <= 128 && stage_count(16, 4) == 8 && stage_count(8, 3) == 9, "stages");

struct MoeParams {
    const uint8_t *x, *router;                   // rows of BF16 or FP16
    uint64_t ld_x, ld_router;                    // elements
    const uint8_t *gate_up_scales, *down_scales;
    uint32_t tokens, experts, top_k, hidden, inter;
    uint32_t hidden_pad, inter_pad;              // rounded up to 64 columns
    uint32_t idesc;                              // matrix instruction without its N
    uint32_t pass;                               // tokens that share a reading of a tile
    uint32_t *ids_out;
    float *weights_out;
    uint8_t *y;
    uint64_t ld_y;                               // elements
    uint32_t spin_limit, skip_copy, skip_math;
    // workspace
    uint32_t *route;                             // [0]: chosen experts, [1]: passes; then the experts' numbers, their first rows and passes
    uint32_t *row_of;                            // [tokens][top_k]: row of a token's j-th expert
    uint32_t *done;                              // [groups of down]: passes of experts whose part is written
    float *h;                                    // [rows][inter_pad]
    float *z;                                    // [rows][hidden_pad]
};

// What a block knows of the routing.
struct Routing {
    uint32_t n_active, n_passes;                 // chosen experts; of up to P.pass tokens each
    uint16_t expert[kMaxExperts];
    uint16_t first[kMaxExperts + 1];             // first row of an expert's tokens
    uint16_t pass[kMaxExperts + 1];              // passes of the experts before
};
struct MoeShared {
    // copied: a stage's weights are there; full: its pieces and scale words are.  Apart, so that a block that gives up can wait for its
    // copies whichever role gave up (0.7 us of the 29 that one token takes).
    uint64_t copied[kMoeMaxStages], full[kMoeMaxStages], empty[kMoeMaxStages], acc_full[2], acc_empty[2];
    uint32_t tmem, failed, unsettled;            // unsettled: copies or matrix instructions that this block did not see the end of
    Routing R;
    alignas(16) float other[2][64][4];           // kernel 1: what the other half of the result warps needs
    float row_p[kMaxRows];
    uint16_t row_of[kMaxRows];                   // kernel 2: rows of the tokens' experts
    uint8_t row_token[kMaxRows];
    uint2 todo[kMoeTodo];                        // kernel 2: first group, and which of its tile's groups, to add up
    uint32_t n_todo;
};
// while routing, where the stages will be
struct MoeRouting {
    float p[kMaxRows];                           // of this block's share of the tokens
    uint16_t id[kMaxRows];
    float p_all[kMaxRows];
    uint16_t id_all[kMaxRows];
    alignas(8) uint32_t mask[2 * kMaxExperts];   // tokens that chose the expert
    uint16_t first_of[kMaxExperts];              // a chosen expert's first row
    // [token, rounded up to 8][expert, to 16]; behind them the warps' sums of logits that several share (there are few then), and
    // columns of router and tokens
    double logits[1];
};
constexpr size_t kMoeSmem = 1024 + kMoeStageSpace + sizeof(MoeShared);
static_assert(sizeof(MoeRouting) + 8 * kMaxExperts * kMaxTokens + (kMaxExperts + kMaxTokens) * 192 + 16 <= kMoeStageSpace && kMoeSmem <= kMaxSmem, "shared memory");

template <bool HALF>
__device__ __forceinline__ void mma16(float c[4], const uint32_t a[4], uint32_t b0, uint32_t b1)
{
    if (HALF) mma_f16(c, a[0], a[1], a[2], a[3], b0, b1);
    else mma_bf16(c, a[0], a[1], a[2], a[3], b0, b1);
}
// ---- the weights' stream --------------------------------------------------------------------------------------------

// A tile: `groups` groups of eight rows (UP: of gate, and behind 64 rows of up) of a chosen expert, for up to P.pass of its tokens.
struct Tile {
    uint32_t expert, group, groups, row, count;  // row, count: its tokens' rows
};

// How the rows of an expert are cut: `per` tiles of `height` groups.
struct Cut { uint32_t height, per; };

// A step of 128 columns takes the block about as long as `kFixed` groups' bytes do even when the tile is small, so blocks want few
// and equal tiles: of all numbers of tiles a block the one whose tiles, as high as they then have to be, take the slowest block least.
template <bool UP>
__device__ __forceinline__ Cut cut_rows(uint32_t rows, uint32_t n_passes, uint32_t blocks)
{
    constexpr uint32_t kMost = UP ? 8 : 16, kFixed = UP ? 4 : 8;
    const uint32_t groups = (rows + 7) >> 3, lane = threadIdx.x & 31;
    const uint32_t least = (n_passes * ((groups + kMost - 1) / kMost) + blocks - 1) / blocks, rounds = least + lane;
    const uint32_t per = min(rounds * blocks / n_passes, groups);
    const uint32_t height = (groups + per - 1) / per;        // per > 0: `least` tiles a block are enough
    const uint32_t cost = rounds * (kFixed + height);
    const uint32_t best = __reduce_min_sync(0xFFFFFFFFu, cost);
    const uint32_t who = __reduce_min_sync(0xFFFFFFFFu, cost == best ? lane : 32u);
    Cut c;
    c.height = __shfl_sync(0xFFFFFFFFu, height, who);
    c.per = (groups + c.height - 1) / c.height;
    return c;
}

// A block's tiles; all roles walk through them alike.  UP: expert by expert.  Down: band of rows by band of rows, in each of them
// expert by expert, so that a band is complete, and its experts can be added up, when a few neighbouring blocks have done with it,
// and not all bands at once at the very end.  The passes over an expert's tokens lie next to each other: the second finds the tile in
// the L2.
template <bool UP>
struct Tiles {
    const Routing& R;
    const Cut cut;
    const uint32_t groups, most;
    uint32_t left, active, band, pass;
    __device__ __forceinline__ Tiles(const Routing& r, const Cut& c, uint32_t rows, uint32_t most_, uint32_t block, uint32_t blocks)
        : R(r), cut(c), groups((rows + 7) >> 3), most(most_), active(0)
    {
        const uint32_t all = c.per * r.n_passes;             // at most 2^13 * 2^10; times the blocks still 32 bits
        const uint32_t first = all * block / blocks;
        left = all * (block + 1) / blocks - first;
        const uint32_t v = UP ? 0 : first % r.n_passes;
        // the last chosen expert whose passes begin at or before the first tile, found by the warp together
        uint32_t before = 0;
        for (uint32_t a = 1 + (threadIdx.x & 31); a < r.n_active; a += 32) before += (UP ? r.pass[a] * c.per <= first : r.pass[a] <= v);
        active = __reduce_add_sync(0xFFFFFFFFu, before);
        if (UP) {
            const uint32_t in = first - r.pass[active] * c.per, n = passes();
            band = in / n;
            pass = in - band * n;
        } else {
            band = first / r.n_passes;
            pass = v - r.pass[active];
        }
    }
    __device__ __forceinline__ uint32_t passes() const { return R.pass[active + 1] - R.pass[active]; }
    __device__ __forceinline__ bool next(Tile& t)
    {
        if (!left) return false;
        --left;
        t.expert = R.expert[active];
        t.group = band * cut.height;
        t.groups = min(cut.height, groups - t.group);
        t.row = R.first[active] + pass * most;
        t.count = min(R.first[active + 1] - t.row, most);
        if (++pass < passes()) return true;
        pass = 0;
        if (UP) {
            if (++band == cut.per) { band = 0; ++active; }
        } else if (++active == R.n_active) {
            active = 0;
            ++band;
        }
        return true;
    }
};

__device__ __forceinline__ uint32_t to_pieces(__half2 v)
{
    return __nv_cvt_halfraw2_to_fp8x2(__half2_raw(v), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ __half2 of_pieces(uint32_t q)
{
    return __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)q, __NV_E4M3));
}

// Four activations of a lane as PIECES E4M3 words, in the block scale of the warp's 128 columns.  FP16 holds what is left behind a
// piece: exactly for BF16 and FP16 activations (EXACT); of FP32 ones it holds what is left behind the second, at most 2^-9 of the value,
// to 2^-12 of that.  What is left behind the pieces before is exact in FP32.
template <int PIECES, bool EXACT>
__device__ __forceinline__ void make_pieces(float v[4], uint32_t words[PIECES], uint32_t& scale)
{
    const uint32_t m01 = max(__float_as_uint(v[0]) & 0x7FFFFFFFu, __float_as_uint(v[1]) & 0x7FFFFFFFu);
    const uint32_t m23 = max(__float_as_uint(v[2]) & 0x7FFFFFFFu, __float_as_uint(v[3]) & 0x7FFFFFFFu);
    uint32_t largest = __reduce_max_sync(0xFFFFFFFFu, max(m01, m23));
    if (largest >= 0x7F800000u) {                // rare: infinities and NaN all become NaN, E4M3 has nothing else
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m = fmaxf(m, finite_abs(v[i]));
            v[i] = fabsf(v[i]) < __int_as_float(0x7F800000) ? v[i] : __int_as_float(0x7FC00000);
        }
        largest = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(m));
    }
    scale = scale_byte<false>(__uint_as_float(largest));
    const float inv = inverse_scale(scale);
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = v[i] * inv;
    const __half2 sixteen = __float2half2_rn(16.0f), minus = __float2half2_rn(-16.0f);
    __half2 a, b;
    if (EXACT) {
        a = __floats2half2_rn(f[0], f[1]);
        b = __floats2half2_rn(f[2], f[3]);
    } else {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(f[0], f[1]), __NV_SATFINITE, __NV_E4M3);
            const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(f[2], f[3]), __NV_SATFINITE, __NV_E4M3);
            words[k] = scale >= 4u * k ? lo | (hi << 16) : 0u;
            const float2 x = __half22float2(of_pieces(lo)), y = __half22float2(of_pieces(hi));
            f[0] = (f[0] - x.x) * 16.0f; f[1] = (f[1] - x.y) * 16.0f;
            f[2] = (f[2] - y.x) * 16.0f; f[3] = (f[3] - y.y) * 16.0f;
        }
        a = __floats2half2_rn(f[0], f[1]);
        b = __floats2half2_rn(f[2], f[3]);
    }
#pragma unroll
    for (int k = EXACT ? 0 : 2; k < PIECES; ++k) {
        const uint32_t lo = to_pieces(a), hi = to_pieces(b);
        // scales end at 2^-127: what would need a smaller one is left out
        words[k] = scale >= 4u * k ? lo | (hi << 16) : 0u;
        if (k + 1 < PIECES) {
            a = __hfma2(of_pieces(lo), minus, __hmul2(a, sixteen));
            b = __hfma2(of_pieces(hi), minus, __hmul2(b, sixteen));
        }
    }
}

// What a block does after the routing: its share of gate and up (UP) or of down.  HALF: activations of gate and up are FP16.
// All threads; they leave it together.
template <bool UP, bool HALF, int PIECES, typename Finish>
__device__ __forceinline__ void stream_weights(const MoeParams& P, const MoeMaps& maps, MoeShared& S, const Cut& cut, uint32_t base, uint32_t blocks, Finish finish)
{
    const uint32_t warp = warp_index(), lane = threadIdx.x & 31;
    const uint32_t cols = UP ? P.hidden : P.inter, rows = UP ? P.inter : P.hidden;
    const uint32_t steps = (cols + 127) >> 7;
    const Waiter wait{P.spin_limit, &S.failed};
    const uint32_t stages = stage_count(P.pass, PIECES), stage_bytes = stage_size(P.pass, PIECES), scales_at = stage_bytes - 1024;
    Tiles<UP> tiles(S.R, cut, rows, P.pass, blockIdx.x, blocks);
    Tile t;
    const uint32_t tmem = S.tmem;
    const uint32_t most = UP ? steps : kPartSteps;
    // the stage of the present step and its round
    uint32_t st = 0, round = 0;
    auto forward = [&] { if (++st == stages) { st = 0; ++round; } };
    auto free_stage = [&] { return round == 0 || wait(smem_u32(&S.empty[st]), (round - 1) & 1); };

    if (warp == 0) {
        bool ok = true;
        while (ok && tiles.next(t)) {
            const uint32_t row0 = t.expert * (UP ? 2 * P.inter : P.hidden) + t.group * 8;
            for (uint32_t k = 0; k < steps; ++k, forward()) {
                if (!(ok = round == 0 || wait.warp(smem_u32(&S.empty[st]), (round - 1) & 1))) break;
                const uint32_t bar = smem_u32(&S.copied[st]), to = base + st * stage_bytes;
                if (elect_one()) {
                    bar_expect(bar, t.groups * (UP ? 2048 : 1024));
                    // as few copies as there are bits in the number of groups: one of 8 rows takes the copy engine as long as one of 64
                    uint32_t i = 0;
#pragma unroll
                    for (int b = UP ? 3 : 4; b >= 0; --b) {
                        if (!(t.groups >> b & 1) || P.skip_copy) continue;
                        tensor_copy<1>(to + i * 1024, &maps.of[b], (int)(k * 128), (int)(row0 + 8 * i), bar);
                        if (UP) tensor_copy<1>(to + 8192 + i * 1024, &maps.of[b], (int)(k * 128), (int)(row0 + P.inter + 8 * i), bar);
                        i += 1u << b;
                    }
                }
                __syncwarp();
            }
        }
        // nothing is copied into this block's shared memory any more, whether the block gave up or not
        if (!P.skip_copy && !settled_stage(smem_u32(S.copied), lane, stages, st, round, P.spin_limit)) S.failed = S.unsettled = 1;
    } else if (warp == 1 && !P.skip_math) {
        uint32_t part = 0, k = steps;            // k: of the present tile, which is done
        bool ok = true;
        while (ok) {
            if (k == steps) {
                if (!tiles.next(t)) break;
                k = 0;
            }
            const uint32_t buf = part & 1, d = tmem + buf * 128, first = k, end = min(steps, k + most);
            const uint32_t idesc = P.idesc | ((piece_rows(t.count, PIECES) >> 3) << 17);
            if (part >= 2 && !(ok = wait.warp(smem_u32(&S.acc_empty[buf]), ((part >> 1) - 1) & 1))) break;
            for (; k < end; ++k, forward()) {
                if (!(ok = wait.warp_both(smem_u32(&S.full[st]), smem_u32(&S.copied[st]), round & 1))) break;
                tc_fence_after();
                const uint32_t at = base + st * stage_bytes, sf = tmem + kMoeTmemScales + st * 8;
                const uint64_t da = operand_desc(at), db = operand_desc(at + 16384);
                if (elect_one()) {
                    tmem_copy_scales<1>(sf, at + scales_at);
                    tmem_copy_scales<1>(sf + 4, at + scales_at + 512);
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j) mma_scaled<1>(d, da + 2 * j, db + 2 * j, idesc, sf, sf + 4, (k - first) | j);
                    mma_commit<1>(smem_u32(&S.empty[st]));
                }
                __syncwarp();
            }
            if (elect_one()) mma_commit<1>(smem_u32(&S.acc_full[buf]));
            __syncwarp();
            ++part;
        }
        // nor do matrix instructions read from there
        if (part && lane == 0 && !settled(smem_u32(&S.acc_full[(part - 1) & 1]), ((part - 1) >> 1) & 1, P.spin_limit)) S.failed = S.unsettled = 1;
    } else if (warp == 2) {
        // scale bytes of the weights, four steps at a time and four steps ahead; row r of the tile's operand is row 32 j + lane
        const uint32_t sld = steps, srows = (rows + 127) >> 7;
        const uint8_t* mine[4];
        auto find_rows = [&] {
            const uint8_t* s = (UP ? P.gate_up_scales + (uint64_t)t.expert * 2 * srows * sld : P.down_scales + (uint64_t)t.expert * srows * sld);
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                const uint32_t r = min((t.group + (UP ? 4 * (j & 1) : 4 * j)) * 8 + lane, rows - 1);
                mine[j] = s + (uint64_t)((UP && j >= 2 ? srows : 0) + (r >> 7)) * sld;
            }
        };
        auto fetch = [&](uint32_t k, uint32_t w[4]) {
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) w[j] = scale_word(mine[j], 0, 0, 0, 1, k, steps);
        };
        uint32_t w[4], ahead[4];
        bool ok = true, more = tiles.next(t);
        if (more) { find_rows(); fetch(0, w); }
        while (ok && more) {
            for (uint32_t k = 0; k < steps && ok; k += 4) {
                if (k + 4 < steps) fetch(k + 4, ahead);
                else if ((more = tiles.next(t))) { find_rows(); fetch(0, ahead); }
                for (uint32_t q = 0; q < 4 && k + q < steps; ++q, forward()) {
                    if (!(ok = __all_sync(0xFFFFFFFFu, free_stage()))) break;
                    const uint32_t at = base + st * stage_bytes + scales_at + lane * 16;
                    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" :: "r"(at), "r"((w[0] >> (8 * q)) & 255u), "r"((w[1] >> (8 * q)) & 255u),
                                 "r"((w[2] >> (8 * q)) & 255u), "r"((w[3] >> (8 * q)) & 255u) : "memory");
                    fence_async_shared();
                    __syncwarp();
                    if (lane == 0) bar_arrive(smem_u32(&S.full[st]));
                }
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j) w[j] = ahead[j];
            }
        }
    } else if (warp >= 8) {
        // a warp has a stage of its own (two have one where there are at most eight): the time of all stages for the latency
        // of its loads, and it sees every phase of its stage's barrier (a wait by parity that skipped one would take the phase
        // before for it)
        const uint32_t sharing = kBuilders / stages, own = (warp - 8) % stages, part = (warp - 8) / stages;
        if (part < sharing) {
            const uint32_t at = base + own * stage_bytes;
            bool ok = true;
            while (ok && tiles.next(t)) {
                const uint32_t padded = (t.count + 7) & ~7u;
                for (uint32_t k = 0; k < steps; ++k, forward()) {
                    if (st != own) continue;
                    const uint32_t col = k * 128 + lane * 4;
                    auto fetch = [&](uint32_t c, uint4 raw[4]) {
#pragma unroll
                        for (uint32_t i = 0; i < 4; ++i) {
                            raw[i] = make_uint4(0, 0, 0, 0);
                            if (c + i >= t.count || col >= cols) continue;
                            if (UP) {
                                const uint8_t* x = P.x + 2 * ((uint64_t)S.row_token[t.row + c + i] * P.ld_x + col);
                                if (col + 4 <= cols) {
                                    const uint2 v = *reinterpret_cast<const uint2*>(x);
                                    raw[i].x = v.x;
                                    raw[i].y = v.y;
                                } else {                     // a row may end where its buffer does
                                    const uint16_t* e = reinterpret_cast<const uint16_t*>(x);
                                    raw[i].x = e[0] | (col + 1 < cols ? (uint32_t)e[1] << 16 : 0u);
                                    raw[i].y = col + 2 < cols ? e[2] : 0u;
                                }
                            } else {
                                raw[i] = *reinterpret_cast<const uint4*>(P.h + (uint64_t)(t.row + c + i) * P.inter_pad + col);
                            }
                        }
                    };
                    // four tokens at a time, whether they are there or not (their rows are): the chain of roundings is long
                    uint4 raw[4], ahead[4];
                    fetch(4 * part, raw);
                    if (!(ok = __all_sync(0xFFFFFFFFu, free_stage()))) break;
                    for (uint32_t c = 4 * part; c < t.count; c += 4 * sharing) {
                        if (c + 4 * sharing < t.count) fetch(c + 4 * sharing, ahead);
#pragma unroll
                        for (uint32_t i = 0; i < 4; ++i) {
                            float v[4];
                            if (UP) {
                                const uint32_t u[2] = {raw[i].x, raw[i].y};
#pragma unroll
                                for (int q = 0; q < 4; ++q) {
                                    const uint16_t s = (uint16_t)(u[q >> 1] >> (16 * (q & 1)));
                                    v[q] = HALF ? __half2float(__ushort_as_half(s)) : __bfloat162float(__ushort_as_bfloat16(s));
                                }
                            } else {
                                v[0] = __uint_as_float(raw[i].x); v[1] = __uint_as_float(raw[i].y);
                                v[2] = __uint_as_float(raw[i].z); v[3] = __uint_as_float(raw[i].w);
                            }
                            if (k + 1 == steps) {
#pragma unroll
                                for (uint32_t q = 0; q < 4; ++q) v[q] = col + q < cols ? v[q] : 0.0f;
                            }
                            uint32_t words[PIECES], scale;
                            make_pieces<PIECES, UP>(v, words, scale);
#pragma unroll
                            for (uint32_t q = 0; q < PIECES; ++q) {
                                const uint32_t r = q * padded + c + i;
                                sts32(at + 16384 + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4, words[q]);
                                if (lane == q) sts32(at + scales_at + 512 + (r & 31) * 16 + (r >> 5) * 4, scale >= 4u * q ? scale - 4u * q : 0u);
                            }
                        }
#pragma unroll
                        for (uint32_t i = 0; i < 4; ++i) raw[i] = ahead[i];
                    }
                    fence_async_shared();
                    __syncwarp();
                    if (lane == 0) bar_arrive(smem_u32(&S.full[st]));
                }
            }
        }
    } else if (warp >= 4) {
        const uint32_t quad = warp & 3;
        uint32_t part = 0, k = steps;
        while (true) {
            if (k == steps) {
                if (!tiles.next(t)) break;
                k = 0;
            }
            const uint32_t buf = part & 1, padded = (t.count + 7) & ~7u;
            // the four warps go on, or stop, together: they meet at a barrier of their own
            uint32_t ok = wait(smem_u32(&S.acc_full[buf]), (part >> 1) & 1) && !*wait.failed;
            asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %0, 0;\n\tbarrier.cta.red.and.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "+r"(ok) :: "memory");
            if (!ok) break;
            tc_fence_after();
            const uint32_t d = tmem + (quad * 32u << 16) + buf * 128;
            for (uint32_t c = 0; c < t.count; c += 8) {
                float piece[PIECES][8];
#pragma unroll
                for (uint32_t q = 0; q < PIECES; ++q) tmem_ld8(d + q * padded + c, piece[q]);
                tmem_ld_wait();
                // the smallest pieces first
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float sum = piece[PIECES - 1][i];
#pragma unroll
                    for (int q = PIECES - 2; q >= 0; --q) sum += piece[q][i];
                    piece[0][i] = sum;
                }
                finish.store(t, c, quad, lane, piece[0], k != 0);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_u32(&S.acc_empty[buf]));
            ++part;
            k = min(steps, k + most);
            if (k == steps) finish.tile_done(t);
        }
    }
    __syncwarp();
    __syncthreads();
    if (threadIdx.x == 0 && S.failed) report(S.unsettled);
}

// ---- routing ----------------------------------------------------------------------------------------------------------

// order of doubles as unsigned numbers, and back; NaN (1) below everything but what is not there (0), both zeros alike
__device__ __forceinline__ unsigned long long order_key(double v)
{
    if (v != v) return 1;
    const unsigned long long b = (unsigned long long)__double_as_longlong(v + 0.0);
    return (b >> 63) ? ~b : b | (1ull << 63);
}
__device__ __forceinline__ double value_of(unsigned long long key)
{
    return key == 1 ? __longlong_as_double(0x7FF8000000000000ll) : __longlong_as_double((long long)((key >> 63) ? key & ~(1ull << 63) : ~key));
}
__device__ __forceinline__ double ld_cluster_f64(uint32_t addr)
{
    double v;
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(addr) : "memory");
    return v;
}

// This block's part of the logits, logits[token][expert]: the cluster's blocks take a share of the columns each, so that a cluster
// reads router and tokens once; they pass through shared memory, from where every warp takes what its 16 experts x 8 tokens need.
// Products of 64 columns are summed by the matrix instructions in FP32, these in FP64: what separates two experts' logits decides
// which weights are used, and 2^-24 of such a sum is far below what the activations' own rounding moves.
template <bool HALF>
__device__ __forceinline__ void router_logits(const MoeParams& P, uint32_t rank, MoeRouting& S)
{
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const uint32_t mt = (P.experts + 15) >> 4, nt = (P.tokens + 7) >> 3, tasks = mt * nt, padded = nt * 8;
    const uint32_t rows_e = mt * 16, rows = rows_e + padded;
    const uint32_t all = (P.hidden + 63) >> 6, lo = all * rank / kMoeCluster, hi = all * (rank + 1) / kMoeCluster;
    uint32_t split = 1;
    while (split * 2 * tasks <= kMoeWarps && split * 2 <= hi - lo) split *= 2;
    double* items = S.logits + rows_e * padded;
    const uint32_t staged = (smem_u32(items + (split > 1 ? kMoeWarps * 128 : 0)) + 15u) & ~15u;
    const uint32_t room = kMoeStageSpace - (staged - smem_u32(&S));
    // columns in pieces of 64 that fit at a time; rows of an odd multiple of 64 bytes keep the 16-byte reads of a warp apart
    const uint32_t fit = min((room / rows - 64) / 128, max(hi - lo, 1u)), pitch = fit * 128 + 64;
    double sum[4] = {0, 0, 0, 0};
    if (split == 1)
        for (uint32_t i = tid; i < rows_e * padded; i += kMoeThreads) S.logits[i] = 0;
    for (uint32_t from = lo; from < hi; from += fit) {
        const uint32_t now = min(fit, hi - from);
        __syncthreads();
        for (uint32_t row = warp; row < rows; row += kMoeWarps) {
            const bool expert = row < rows_e;
            const uint32_t r = expert ? row : row - rows_e;
            const bool there = r < (expert ? P.experts : P.tokens);
            const uint8_t* src = !there ? P.x : expert ? P.router + 2 * (uint64_t)r * P.ld_router : P.x + 2 * (uint64_t)r * P.ld_x;
            for (uint32_t piece = lane; piece < now * 8; piece += 32) {
                const uint32_t col = from * 64 + piece * 8;
                const bool in = there && col < P.hidden;
                async_copy16(staged + row * pitch + piece * 16, in ? src + 2 * col : P.x, in ? min(16u, 2 * (P.hidden - col)) : 0u);
            }
        }
        async_copy_wait();
        __syncthreads();
        for (uint32_t item = warp; item < tasks * split; item += kMoeWarps) {
            const uint32_t task = item / split, slice = item - task * split, e0 = (task / nt) * 16, k0 = (task % nt) * 8;
            const uint32_t ra = staged + (e0 + g) * pitch + 16 * t, rb = ra + 8 * pitch, rx = staged + (rows_e + k0 + g) * pitch + 16 * t;
            double s[4] = {0, 0, 0, 0};
            for (uint32_t u = now * slice / split; u < now * (slice + 1) / split; ++u) {
                float v[4] = {0, 0, 0, 0};
#pragma unroll
                for (uint32_t j = 0; j < 2; ++j) {
                    const uint4 a = lds128(ra + u * 128 + j * 64), b = lds128(rb + u * 128 + j * 64), x = lds128(rx + u * 128 + j * 64);
                    const uint32_t first[4] = {a.x, b.x, a.y, b.y}, second[4] = {a.z, b.z, a.w, b.w};
                    mma16<HALF>(v, first, x.x, x.y);
                    mma16<HALF>(v, second, x.z, x.w);
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) s[q] += (double)v[q];
            }
#pragma unroll
            for (uint32_t q = 0; q < 4; ++q) {
                if (split > 1) sum[q] += s[q];               // a warp has one item at most
                else S.logits[(k0 + 2 * t + (q & 1)) * rows_e + e0 + g + 8 * (q >> 1)] += s[q];
            }
        }
    }
    if (split == 1) return;
    if (warp < tasks * split) {
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q) items[warp * 128 + q * 32 + lane] = sum[q];
    }
    __syncthreads();
    for (uint32_t i = tid; i < tasks * 128; i += kMoeThreads) {
        const uint32_t task = i >> 7, q = (i >> 5) & 3, l = i & 31;
        double s = 0;
        for (uint32_t k = 0; k < split; ++k) s += items[(task * split + k) * 128 + q * 32 + l];
        S.logits[((task % nt) * 8 + 2 * (l & 3) + (q & 1)) * rows_e + (task / nt) * 16 + (l >> 2) + 8 * (q >> 1)] = s;
    }
}

// The top_k experts and their weights for this block's share of the tokens (rank, rank + 4, ...), one warp a token.
__device__ __forceinline__ void choose(const MoeParams& P, uint32_t rank, MoeRouting& S)
{
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t base = smem_u32(S.logits), rows_e = (P.experts + 15) & ~15u;
    for (uint32_t i = warp; rank + i * kMoeCluster < P.tokens; i += kMoeWarps) {
        const uint32_t tok = rank + i * kMoeCluster;
        unsigned long long key[kMaxExperts / 32];
        const uint32_t words = (P.experts + 31) >> 5;
#pragma unroll
        for (uint32_t k = 0; k < kMaxExperts / 32; ++k) {
            const uint32_t e = k * 32 + lane;
            key[k] = 0;
            if (e < P.experts) {
                double v = 0;
#pragma unroll
                for (uint32_t r = 0; r < kMoeCluster; ++r) v += ld_cluster_f64(map_shared(base + 8 * (tok * rows_e + e), r));
                key[k] = order_key(v);
            }
        }
        // lane j keeps the j-th choice
        double largest = 0;
        float total = 0, mine = 0;
        uint32_t my_id = 0;
        for (uint32_t j = 0; j < P.top_k; ++j) {
            unsigned long long best = key[0];
            uint32_t where = 0;
#pragma unroll
            for (uint32_t k = 1; k < kMaxExperts / 32; ++k) {
                if (k >= words) break;
                if (key[k] > best) { best = key[k]; where = k; }
            }
            const uint32_t hi = __reduce_max_sync(0xFFFFFFFFu, (uint32_t)(best >> 32));
            const uint32_t lo = __reduce_max_sync(0xFFFFFFFFu, (uint32_t)(best >> 32) == hi ? (uint32_t)best : 0u);
            const bool tie = (uint32_t)(best >> 32) == hi && (uint32_t)best == lo;
            const uint32_t e = __reduce_min_sync(0xFFFFFFFFu, tie ? where * 32 + lane : 0xFFFFFFFFu);
#pragma unroll
            for (uint32_t k = 0; k < kMaxExperts / 32; ++k) {
                if (k >= words) break;
                if (k * 32 + lane == e) key[k] = 0;
            }
            const double v = value_of(((unsigned long long)hi << 32) | lo);
            if (j == 0) largest = v;
            const float p = expf((float)(v - largest));      // the difference in FP64, the exponential in FP32
            total += p;
            if (lane == j) { mine = p; my_id = e; }
        }
        if (lane < P.top_k) {
            S.id[i * P.top_k + lane] = (uint16_t)my_id;
            S.p[i * P.top_k + lane] = mine / total;
        }
    }
}

// From the tokens' choices to the experts' lists: tokens of an expert in ascending order, experts in ascending order.
__device__ __forceinline__ void make_lists(const MoeParams& P, MoeRouting& S, Routing& R)
{
    const uint32_t tid = threadIdx.x, n = P.tokens * P.top_k;
    for (uint32_t e = tid; e < 2 * kMaxExperts; e += kMoeThreads) S.mask[e] = 0;
    __syncthreads();
    for (uint32_t i = tid; i < n; i += kMoeThreads) {
        const uint32_t tok = i / P.top_k;
        atomicOr(&S.mask[2 * S.id_all[i] + (tok >> 5)], 1u << (tok & 31));
    }
    __syncthreads();
    if (tid < 32) {
        // each lane eight experts: counts of tokens, of chosen experts, of passes; sums over the lanes before
        uint32_t count[8], tokens = 0, active = 0, passes = 0;
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) {
            const uint2 m = *reinterpret_cast<const uint2*>(&S.mask[2 * (tid * 8 + k)]);
            count[k] = __popc(m.x) + __popc(m.y);
            tokens += count[k];
            active += count[k] != 0;
            passes += (count[k] + P.pass - 1) / P.pass;
        }
        uint32_t a = tokens, b = active, c = passes;
        for (uint32_t d = 1; d < 32; d <<= 1) {
            const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, a, d), y = __shfl_up_sync(0xFFFFFFFFu, b, d), z = __shfl_up_sync(0xFFFFFFFFu, c, d);
            if (tid >= d) { a += x; b += y; c += z; }
        }
        uint32_t row = a - tokens, at = b - active, pass = c - passes;
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) {
            if (!count[k]) continue;
            R.expert[at] = (uint16_t)(tid * 8 + k);
            R.first[at] = (uint16_t)row;
            R.pass[at] = (uint16_t)pass;
            S.first_of[tid * 8 + k] = (uint16_t)row;
            ++at;
            row += count[k];
            pass += (count[k] + P.pass - 1) / P.pass;
        }
        if (tid == 31) {
            R.n_active = b;
            R.n_passes = c;
            R.first[b] = (uint16_t)a;
            R.pass[b] = (uint16_t)c;
        }
    }
    __syncthreads();
}

// Row of a token in the list of an expert that it chose.
__device__ __forceinline__ uint32_t row_of(const MoeRouting& S, uint32_t e, uint32_t token)
{
    const uint32_t lo = S.mask[2 * e], hi = S.mask[2 * e + 1], below = (1u << (token & 31)) - 1u;
    return S.first_of[e] + (token < 32 ? __popc(lo & below) : __popc(lo) + __popc(hi & below));
}

// Barriers and tensor memory; all threads.
__device__ __forceinline__ void moe_setup(MoeShared& S, uint32_t sharing)
{
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (warp == 0) {
        if (lane < kMoeMaxStages) { bar_init(smem_u32(&S.copied[lane]), 1); bar_init(smem_u32(&S.full[lane]), 1 + sharing); bar_init(smem_u32(&S.empty[lane]), 1); }
        if (lane < 2) { bar_init(smem_u32(&S.acc_full[lane]), 1); bar_init(smem_u32(&S.acc_empty[lane]), 4); }
        if (lane == 0) S.failed = S.unsettled = S.n_todo = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        __syncwarp();
    }
    if (warp == 1) tmem_alloc<1>(smem_u32(&S.tmem), kMoeTmemCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
}

// silu(gate) * up * p into the hidden vectors.  Warps 0 and 1 have the gates, 2 and 3 the ups of the same channels: each half
// gives the other what it needs of every second half of the tokens through shared memory.
struct FinishUp {
    const MoeParams& P;
    MoeShared& S;
    __device__ __forceinline__ void store(const Tile& t, uint32_t c, uint32_t quad, uint32_t lane, const float v[8], bool) const
    {
        const uint32_t row = (quad & 1) * 32 + lane, ch = t.group * 8 + row, mine = quad >> 1;     // gates' warps take tokens 0-3, ups' 4-7
        float* out = S.other[mine ^ 1][row];
        *reinterpret_cast<float4*>(out) = mine ? make_float4(v[0], v[1], v[2], v[3]) : make_float4(v[4], v[5], v[6], v[7]);
        asm volatile("bar.sync 1, 128;" ::: "memory");
        const float4 x = *reinterpret_cast<const float4*>(S.other[mine][row]);
        const float o[4] = {x.x, x.y, x.z, x.w};
        asm volatile("bar.sync 1, 128;" ::: "memory");
        if (row < t.groups * 8 && ch < P.inter) {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                const uint32_t n = c + 4 * mine + i;
                const float gate = mine ? o[i] : v[i], up = mine ? v[4 + i] : o[i];
                if (n < t.count) P.h[(uint64_t)(t.row + n) * P.inter_pad + ch] = gate / (1.0f + expf(-gate)) * up * S.row_p[t.row + n];
            }
        }
    }
    __device__ __forceinline__ void tile_done(const Tile&) const { }
};

template <bool HALF>
struct FinishDown {
    const MoeParams& P;
    MoeShared& S;
    uint32_t n_passes;
    __device__ __forceinline__ void store(const Tile& t, uint32_t c, uint32_t quad, uint32_t lane, const float v[8], bool add) const
    {
        const uint32_t row = quad * 32 + lane, r = t.group * 8 + row;
        if (row >= t.groups * 8 || r >= P.hidden) return;
        float* z = P.z + (uint64_t)(t.row + c) * P.hidden_pad + r;
        float sum[8];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) sum[i] = c + i < t.count && add ? v[i] + z[(uint64_t)i * P.hidden_pad] : v[i];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (c + i < t.count) z[(uint64_t)i * P.hidden_pad] = sum[i];
    }
    // The four warps: whoever completes a group's last pass adds its experts up, at the end, with all of the block's threads (they wait
    // for little but loads then: 128 threads took 16 us after the last product of 64 tokens).
    __device__ __forceinline__ void tile_done(const Tile& t) const
    {
        const uint32_t tid = threadIdx.x & 127;
        __threadfence();
        asm volatile("bar.sync 1, 128;" ::: "memory");
        if (tid < 32) {
            const bool last = tid < t.groups && atomicAdd(&P.done[t.group + tid], 1u) + 1 == n_passes;
            const uint32_t which = __ballot_sync(0xFFFFFFFFu, last);
            __threadfence();
            if (tid == 0 && which) {
                S.todo[S.n_todo] = make_uint2(t.group, which);
                ++S.n_todo;
            }
        }
    }
    // Thread tid of n: four columns of a token at a time.
    __device__ __forceinline__ void add_up(uint32_t tid, uint32_t n) const
    {
        const uint32_t todo = S.n_todo, per = 32 * P.tokens;
        for (uint32_t i = tid; i < todo * per; i += n) {
            const uint32_t k = i / per, in = i - k * per, tok = in >> 5, g = (in & 31) >> 1;
            const uint2 what = S.todo[k];
            const uint32_t r = (what.x + g) * 8 + (in & 1) * 4;
            if (!(what.y >> g & 1) || r >= P.hidden) continue;
            float y[4] = {0, 0, 0, 0};
            const uint16_t* rows = S.row_of + tok * P.top_k;
#pragma unroll 8
            for (uint32_t j = 0; j < P.top_k; ++j) {
                const float4 z = __ldcg(reinterpret_cast<const float4*>(P.z + (uint64_t)rows[j] * P.hidden_pad + r));
                y[0] += z.x; y[1] += z.y; y[2] += z.z; y[3] += z.w;
            }
#pragma unroll
            for (uint32_t q = 0; q < 4; ++q) {
                if (r + q >= P.hidden) break;
                if (HALF) reinterpret_cast<__half*>(P.y)[(uint64_t)tok * P.ld_y + r + q] = __float2half_rn(y[q]);
                else reinterpret_cast<__nv_bfloat16*>(P.y)[(uint64_t)tok * P.ld_y + r + q] = __float2bfloat16_rn(y[q]);
            }
        }
    }
};

// Hidden vectors, FP32 in memory, go into the product as four pieces: 2^-19 of the value and 2^-21 for what FP16 holds of it, a
// thousandth of half a step of y in BF16, a hundredth in FP16.  (Three pieces of BF16 layers left 2^-14: y of 64 tokens and 64 experts was
// 2.5e-4 from that of an FP32 form, 7.3e-5 with four, both in 119 us: the builders have the time.)
constexpr int kHiddenPieces = 4;

template <bool HALF>
__global__ void __launch_bounds__(kMoeThreads, 1)
moe_up_kernel(const __grid_constant__ MoeMaps maps, const __grid_constant__ MoeParams P)
{
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    uint8_t* aligned = raw + (base - smem_u32(raw));
    MoeShared& S = *reinterpret_cast<MoeShared*>(aligned + kMoeStageSpace);
    MoeRouting& T = *reinterpret_cast<MoeRouting*>(aligned);
    const uint32_t tid = threadIdx.x, rank = cluster_rank();
    const uint32_t n_rows = P.tokens * P.top_k;

    if (tid < kMoeHeights) prefetch_map(&maps.of[tid]);
    moe_setup(S, kBuilders / stage_count(P.pass, 3));
    grid_wait();
    grid_launch_dependents();
    router_logits<HALF>(P, rank, T);
    cluster_sync();
    choose(P, rank, T);
    cluster_sync();
    for (uint32_t i = tid; i < n_rows; i += kMoeThreads) {
        const uint32_t tok = i / P.top_k, j = i % P.top_k, at = (tok / kMoeCluster) * P.top_k + j, from = tok % kMoeCluster;
        float p;
        uint16_t id;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(p) : "r"(map_shared(smem_u32(&T.p[at]), from)) : "memory");
        asm volatile("ld.shared::cluster.u16 %0, [%1];" : "=h"(id) : "r"(map_shared(smem_u32(&T.id[at]), from)) : "memory");
        T.p_all[i] = p;
        T.id_all[i] = id;
    }
    make_lists(P, T, S.R);
    for (uint32_t i = tid; i < n_rows; i += kMoeThreads) {
        const uint32_t r = row_of(T, T.id_all[i], i / P.top_k);
        S.row_p[r] = T.p_all[i];
        S.row_token[r] = (uint8_t)(i / P.top_k);
        if (blockIdx.x == 0) {
            P.row_of[i] = r;
            if (P.ids_out) P.ids_out[i] = T.id_all[i];
            if (P.weights_out) P.weights_out[i] = T.p_all[i];
        }
    }
    if (blockIdx.x == 0) {
        for (uint32_t i = tid; i < (P.hidden + 7) / 8; i += kMoeThreads) P.done[i] = 0;
        for (uint32_t i = tid; i <= S.R.n_active; i += kMoeThreads) {
            if (i < S.R.n_active) P.route[2 + i] = S.R.expert[i];
            P.route[2 + kMaxExperts + i] = (uint32_t)S.R.first[i] | ((uint32_t)S.R.pass[i] << 16);
        }
        if (tid == 0) { P.route[0] = S.R.n_active; P.route[1] = S.R.n_passes; }
    }
    fence_async_shared();                        // the routing's shared memory becomes the stages'
    cluster_sync();                              // and no other block reads from it any more
    stream_weights<true, HALF, 3>(P, maps, S, cut_rows<true>(P.inter, S.R.n_passes, gridDim.x), base, gridDim.x, FinishUp{P, S});
    if (tid < 64 && tid >= 32) tmem_free<1>(S.tmem, kMoeTmemCols);
}

template <bool HALF>
__global__ void __launch_bounds__(kMoeThreads, 1)
moe_down_kernel(const __grid_constant__ MoeMaps maps, const __grid_constant__ MoeParams P)
{
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    MoeShared& S = *reinterpret_cast<MoeShared*>(raw + (base - smem_u32(raw)) + kMoeStageSpace);
    const uint32_t tid = threadIdx.x;
    if (tid < kMoeHeights) prefetch_map(&maps.of[tid]);
    moe_setup(S, kBuilders / stage_count(P.pass, kHiddenPieces));
    grid_wait();
    grid_launch_dependents();
    // all of the lists at once, whatever is behind the last chosen expert: one latency
    const uint32_t n_active = P.route[0], n_passes = P.route[1];
    if (tid <= kMaxExperts) {
        const uint32_t v = P.route[2 + kMaxExperts + tid];
        if (tid < kMaxExperts) S.R.expert[tid] = (uint16_t)P.route[2 + tid];
        S.R.first[tid] = (uint16_t)v;
        S.R.pass[tid] = (uint16_t)(v >> 16);
    }
    for (uint32_t i = tid; i < P.tokens * P.top_k; i += kMoeThreads) S.row_of[i] = (uint16_t)P.row_of[i];
    if (tid == 0) { S.R.n_active = n_active; S.R.n_passes = n_passes; }
    __syncthreads();
    const FinishDown<HALF> finish{P, S, n_passes};
    stream_weights<false, HALF, kHiddenPieces>(P, maps, S, cut_rows<false>(P.hidden, n_passes, gridDim.x), base, gridDim.x, finish);
    finish.add_up(tid, kMoeThreads);
    __syncthreads();
    if (tid < 64 && tid >= 32) tmem_free<1>(S.tmem, kMoeTmemCols);
}

// ---- host ----

struct MoeLayout { size_t route, row_of, done, h, z, total; };
static MoeLayout moe_layout(const zc_fp8_moe_layer* L, uint32_t tokens)
{
    const uint64_t rows = (uint64_t)tokens * L->top_k, inter_pad = round_up(L->inter, 64), hidden_pad = round_up(L->hidden, 64);
    MoeLayout o{};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += round_up(bytes, 256); return here; };
    o.route = take(4 * (2 + 2 * kMaxExperts + 2));
    o.row_of = take(4 * rows);
    o.done = take(4 * (hidden_pad / 8));
    o.h = take(4 * rows * inter_pad);
    o.z = take(4 * rows * hidden_pad);
    o.total = at;
    return o;
}

static zc_status check_layer(const zc_fp8_moe_layer* L, uint32_t tokens)
{
    if (!L) return ZC_E_INVALID_ARG;
    if (!fp8_format(L->format) || (L->real_type != ZC_REAL_BF16 && L->real_type != ZC_REAL_F16)) return ZC_E_UNSUPPORTED;
    if (!L->n_experts || !L->top_k || L->top_k > L->n_experts || !L->hidden || !L->inter) return ZC_E_INVALID_ARG;
    if (tokens > kMaxTokens || L->n_experts > kMaxExperts || L->top_k > ZC_FP8_MOE_MAX_TOP_K || L->hidden > 65536 || L->inter > 65536) return ZC_E_TOO_LARGE;
    if (!L->d_router || !L->d_gate_up || !L->d_gate_up_scales || !L->d_down || !L->d_down_scales) return ZC_E_INVALID_ARG;
    if (!aligned16(L->d_router) || !aligned16(L->d_gate_up) || !aligned16(L->d_down)) return ZC_E_INVALID_ARG;
    if (L->ld_router < L->hidden || L->ld_router % 8 || L->ld_gate_up < L->hidden || L->ld_gate_up % 16 || L->ld_down < L->inter || L->ld_down % 16) return ZC_E_INVALID_ARG;
    if (L->ld_router >= (1ull << 32) || L->ld_gate_up >= (1ull << 32) || L->ld_down >= (1ull << 32)) return ZC_E_INVALID_ARG;
    return ZC_OK;
}

// Blocks of `kernel` that are on the GPU at once, in whole clusters: one per SM where clusters of four fill it.
static uint32_t resident_blocks(const void* kernel, uint32_t cluster)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((uint32_t)sm_count() / cluster * cluster);
    cfg.blockDim = dim3(kMoeThreads);
    cfg.dynamicSmemBytes = kMoeSmem;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {cluster, 1, 1};
    cfg.attrs = at;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n <= 0) return 0;
    return std::min((uint32_t)n * cluster, cfg.gridDim.x);
}

template <bool HALF>
static cudaError_t launch_moe(const MoeMaps& up, const MoeMaps& down, const MoeParams& P, cudaStream_t st)
{
    cudaError_t e = cudaSuccess;
    static OncePerDevice once;
    const uint32_t up_blocks = once([&]() -> uint32_t {
        if (cudaFuncSetAttribute(moe_up_kernel<HALF>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMoeSmem) != cudaSuccess) return 0;
        if (cudaFuncSetAttribute(moe_down_kernel<HALF>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMoeSmem) != cudaSuccess) return 0;
        return resident_blocks((const void*)moe_up_kernel<HALF>, kMoeCluster);
    });
    if (!up_blocks || sm_count() < 32) return cudaErrorUnknown;
    cudaLaunchConfig_t cfg{};
    cfg.blockDim = dim3(kMoeThreads);
    cfg.dynamicSmemBytes = kMoeSmem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0] = launch_early();
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim = {kMoeCluster, 1, 1};
    cfg.attrs = at;
    cfg.numAttrs = 2;
    cfg.gridDim = dim3(up_blocks);
    e = cudaLaunchKernelEx(&cfg, moe_up_kernel<HALF>, up, P);
    if (e != cudaSuccess) return e;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3((uint32_t)sm_count());
    return cudaLaunchKernelEx(&cfg, moe_down_kernel<HALF>, down, P);
}

unsigned int* moe_marks_word() { return marks_word(); }

}  // namespace zc

using namespace zc;

extern "C" {

size_t zc_fp8_moe_workspace_bytes(const zc_fp8_moe_layer* layer, uint32_t n_tokens)
{
    return check_layer(layer, n_tokens) == ZC_OK ? moe_layout(layer, n_tokens).total : 0;
}

zc_status zc_fp8_moe(const zc_fp8_moe_layer* layer, uint32_t n_tokens, const void* d_x, uint64_t ld_x, void* d_out, uint64_t ld_out,
                     uint32_t* d_ids, float* d_weights, void* d_workspace, size_t workspace_bytes, void* cuda_stream)
{
    if (const zc_status s = check_layer(layer, n_tokens)) return s;
    if (n_tokens == 0) return ZC_OK;
    if (!d_x || !aligned16(d_x) || ld_x < layer->hidden || ld_x % 8 || ld_x >= (1ull << 32)) return ZC_E_INVALID_ARG;
    if (!d_out || reinterpret_cast<uintptr_t>(d_out) % 2 || ld_out < layer->hidden || ld_out >= (1ull << 32)) return ZC_E_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(d_ids) % 4 || reinterpret_cast<uintptr_t>(d_weights) % 4) return ZC_E_INVALID_ARG;
    if (!d_workspace || reinterpret_cast<uintptr_t>(d_workspace) % 256) return ZC_E_INVALID_ARG;
    const MoeLayout o = moe_layout(layer, n_tokens);
    if (workspace_bytes < o.total) return ZC_E_BUFFER_TOO_SMALL;
    uint8_t* ws = (uint8_t*)d_workspace;
    MoeParams P{};
    P.x = (const uint8_t*)d_x;
    P.router = (const uint8_t*)layer->d_router;
    P.ld_x = ld_x;
    P.ld_router = layer->ld_router;
    P.gate_up_scales = (const uint8_t*)layer->d_gate_up_scales;
    P.down_scales = (const uint8_t*)layer->d_down_scales;
    P.idesc = instruction_of(layer->format, ZC_FMT_FP8_E4M3, 128, 0);
    // Tokens per reading of a tile: the stages that hold their pieces get larger and fewer with them (9 of 8 tokens, 8 of 16, 6 or 7 of 32), an expert
    // that more tokens chose is read again, from the L2.  64 tokens, 2048 / 1024: with 64 experts, top 8, 117 us in passes of 16, 131 of 8, 125 of
    // 32; with 32 experts, top 8 (16 an expert), 93, 114 and 103; with 16, top 4, 62.8, 71 and 66.
    P.pass = n_tokens <= 8 ? 8 : 16;
    P.spin_limit = test_knobs().spin_limit;
    P.skip_copy = test_knobs().skip_copy;
    P.skip_math = test_knobs().skip_math;
    P.tokens = n_tokens;
    P.experts = layer->n_experts;
    P.top_k = layer->top_k;
    P.hidden = layer->hidden;
    P.inter = layer->inter;
    P.hidden_pad = (uint32_t)round_up(layer->hidden, 64);
    P.inter_pad = (uint32_t)round_up(layer->inter, 64);
    P.ids_out = d_ids;
    P.weights_out = d_weights;
    P.y = (uint8_t*)d_out;
    P.ld_y = ld_out;
    P.route = (uint32_t*)(ws + o.route);
    P.row_of = (uint32_t*)(ws + o.row_of);
    P.done = (uint32_t*)(ws + o.done);
    P.h = (float*)(ws + o.h);
    P.z = (float*)(ws + o.z);
    MoeMaps up, down;
    for (uint32_t b = 0; b < kMoeHeights; ++b)
        if (!make_map(&up.of[b], layer->d_gate_up, (uint64_t)layer->n_experts * 2 * layer->inter, layer->hidden, layer->ld_gate_up, 8u << b) ||
            !make_map(&down.of[b], layer->d_down, (uint64_t)layer->n_experts * layer->hidden, layer->inter, layer->ld_down, 8u << b)) return ZC_E_CUDA;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const cudaError_t e = layer->real_type == ZC_REAL_F16 ? launch_moe<true>(up, down, P, st) : launch_moe<false>(up, down, P, st);
    return e == cudaSuccess ? ZC_OK : ZC_E_CUDA;
}

}  // extern "C"
