// zc_fp8_moe: a mixture-of-experts layer for a few tokens, in two kernels.
//
// With a few tokens the time goes into reading the chosen experts' weights once.  They are streamed by tensor copies into shared
// memory and multiplied there as they are, FP8 with their scale bytes, on the fifth-generation tensor cores: no thread ever
// touches a weight.  (Widening them in registers for warp-wide BF16 instructions took 350 instructions per KiB and ran at a
// sixth of the memory's rate.)  The instruction wants FP8 on the other side as well, so an activation is written as a sum of
// E4M3 pieces, v = 2^s (q0 + 2^-4 q1 + 2^-8 q2 + ...), with s from the largest magnitude of 128 columns: q_i is what the
// pieces before it leave, rounded, and each piece takes at least four bits more.  Three pieces hold BF16 and FP16 exactly
// (8 and 11 bits) down to 2^-17 of the largest of the 128, and nothing smaller is off by more than 2^-25 of it.  The
// pieces are rows of the same operand, so they cost columns of the accumulator, and their sum is taken in FP32 at the end.
//
// Rows are handed out in groups of eight, the swizzle's height: tiles of all chosen experts form one sequence of groups that is cut
// into equal ranges, one per block.
//
//   kernel 1  routes (every cluster for itself, so that no block waits for another cluster), then gate and up: a tile is up to 64
//             rows of gate and the same of up in alternating groups, so that a warp ends with both
//   kernel 2  down: up to 128 rows a tile, one FP32 row of partial results per (token, expert); the block that completes a
//             group's last expert adds the experts up in the order of the token's list
//
// Warps of a block: 0 tensor copies, 1 matrix instructions, 2 the weights' scale bytes, 4-7 results, 8-13 the activations' pieces (14, 15: routing only).
#include "zc_fp8_tensor.cuh"

namespace zc {

constexpr uint32_t kMoeWarps = 16, kMoeThreads = 32 * kMoeWarps;
constexpr uint32_t kMoeCluster = 4;
constexpr uint32_t kMoePass = 32;                // tokens that share a reading of a tile
constexpr uint32_t kMaxTokens = ZC_FP8_MOE_MAX_TOKENS, kMaxExperts = ZC_FP8_MOE_MAX_EXPERTS;
constexpr uint32_t kMaxRows = kMaxTokens * ZC_FP8_MOE_MAX_TOP_K;
constexpr uint32_t kMoeStages = 6;
constexpr uint32_t kMoeStageBytes = 16384 + 16384 + 1024 + 1024;   // weights, pieces, scale words of both (the rest keeps 1 KiB alignment)
constexpr uint32_t kMoeHeights = 5;              // tensor copies of 8, 16, 32, 64 and 128 rows
constexpr uint32_t kMoeTmemCols = 512;           // two accumulators of 128 columns, then 4 + 4 scale columns per stage
constexpr uint32_t kMoeTmemScales = 256;

struct MoeMaps { CUtensorMap of[kMoeHeights]; };

struct MoeParams {
    const uint8_t *x, *router;                   // rows of BF16 or FP16
    uint64_t ld_x, ld_router;                    // elements
    const uint8_t *gate_up_scales, *down_scales;
    uint32_t tokens, experts, top_k, hidden, inter;
    uint32_t hidden_pad, inter_pad;              // rounded up to 64 columns
    uint32_t idesc;                              // matrix instruction without its N
    uint32_t *ids_out;
    float *weights_out;
    uint8_t *y;
    uint64_t ld_y;                               // elements
    uint32_t spin_limit, skip_copy;
    // workspace
    uint32_t *route;                             // [0]: chosen experts, [1]: passes; then the experts' numbers, their first rows and passes
    uint32_t *row_of;                            // [tokens][top_k]: row of a token's j-th expert
    uint32_t *done;                              // [groups of down]: passes of experts whose part is written
    float *h;                                    // [rows][inter_pad]
    float *z;                                    // [rows][hidden_pad]
};

// What a block knows of the routing.
struct Routing {
    uint32_t n_active, n_passes;                 // chosen experts; of up to 32 tokens each
    uint16_t expert[kMaxExperts];
    uint16_t first[kMaxExperts + 1];             // first row of an expert's tokens
    uint16_t pass[kMaxExperts + 1];              // passes of the experts before
};
struct MoeShared {
    uint64_t full[kMoeStages], empty[kMoeStages], acc_full[2], acc_empty[2];
    uint32_t tmem, failed;
    Routing R;
    alignas(16) float other[2][64][4];           // kernel 1: what the other half of the result warps needs
    float row_p[kMaxRows];
    uint16_t row_of[kMaxRows];                   // kernel 2: rows of the tokens' experts
    uint8_t row_token[kMaxRows];
    uint32_t last[16];
};
// while routing, where the stages will be
struct MoeRouting {
    double items[16 * 128], logits[kMaxExperts * kMaxTokens];
    float p[kMaxRows];                           // of this block's share of the tokens
    uint16_t id[kMaxRows];
    float p_all[kMaxRows];
    uint16_t id_all[kMaxRows];
    unsigned long long mask[kMaxExperts];        // tokens that chose the expert
};
constexpr size_t kMoeSmem = 1024 + kMoeStages * kMoeStageBytes + sizeof(MoeShared);
static_assert(sizeof(MoeRouting) <= kMoeStages * kMoeStageBytes && kMoeSmem <= kMaxSmem, "shared memory");

template <bool HALF>
__device__ __forceinline__ void mma16(float c[4], const uint32_t a[4], uint32_t b0, uint32_t b1)
{
    if (HALF) mma_f16(c, a[0], a[1], a[2], a[3], b0, b1);
    else mma_bf16(c, a[0], a[1], a[2], a[3], b0, b1);
}
// the first n bytes of a 16-byte piece, the rest as zeros
__device__ __forceinline__ uint4 first_bytes(uint4 v, uint32_t n)
{
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const uint32_t have = n > 4 * i ? n - 4 * i : 0;
        if (have < 4) w[i] &= (1u << (8 * have)) - 1u;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 ld_cached_v4(const void* p) { return __ldg(reinterpret_cast<const uint4*>(p)); }
__device__ __forceinline__ uint4 zero4() { return make_uint4(0, 0, 0, 0); }

// ---- the weights' stream --------------------------------------------------------------------------------------------

// A tile: `groups` groups of eight rows (UP: of gate, and behind 64 rows of up) of a chosen expert, for up to 32 of its tokens.
struct Tile {
    uint32_t active, expert, group, groups, row, count;      // row, count: its tokens' rows
};

// The tiles of units first .. end - 1; all roles walk through them alike.  A unit is a group of an expert.  UP: expert by
// expert.  Down: bands of 128 rows, in each of them expert by expert, so that a band is complete, and its experts can be added up, when a
// few neighbouring blocks have done with it, and not all bands at once at the very end.
template <bool UP>
struct Tiles {
    static constexpr uint32_t kMost = UP ? 8 : 16;
    const Routing& R;
    uint32_t groups, at, end, pass;
    __device__ __forceinline__ Tiles(const Routing& r, uint32_t rows, uint32_t block, uint32_t blocks)
        : R(r), groups((rows + 7) >> 3), pass(0)
    {
        const uint64_t units = (uint64_t)groups * r.n_active;
        at = (uint32_t)(units * block / blocks);
        end = (uint32_t)(units * (block + 1) / blocks);
    }
    __device__ __forceinline__ bool next(Tile& t)
    {
        if (at >= end) return false;
        uint32_t left;
        if (UP) {
            t.active = at / groups;
            t.group = at - t.active * groups;
            left = min(end - at, groups - t.group);
            // a remainder is shared by the last two tiles
            t.groups = left > kMost && left < 2 * kMost ? (left + 1) / 2 : min(left, kMost);
        } else {
            const uint32_t band = at / (kMost * R.n_active), first = band * kMost, height = min(groups - first, kMost);
            const uint32_t in = at - first * R.n_active;
            t.active = in / height;
            t.group = first + in - t.active * height;
            t.groups = min(end - at, first + height - t.group);
        }
        t.expert = R.expert[t.active];
        t.row = R.first[t.active] + pass * kMoePass;
        const uint32_t n = R.first[t.active + 1] - t.row;
        t.count = min(n, kMoePass);
        if (n > kMoePass) ++pass;
        else { pass = 0; at += t.groups; }
        return true;
    }
};

// Four activations of a lane as PIECES E4M3 words, in the block scale of the warp's 128 columns.
template <int PIECES>
__device__ __forceinline__ void make_pieces(const float v[4], uint32_t words[PIECES], uint32_t& scale)
{
    float m = fmaxf(fmaxf(finite_abs(v[0]), finite_abs(v[1])), fmaxf(finite_abs(v[2]), finite_abs(v[3])));
    m = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(m)));
    scale = scale_byte<false>(m);
    const float inv = inverse_scale(scale);
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = fabsf(v[i]) < __int_as_float(0x7F800000) ? v[i] * inv : __int_as_float(0x7FC00000);   // E4M3 has no infinity
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(f[0], f[1]), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(f[2], f[3]), __NV_SATFINITE, __NV_E4M3);
        // scales end at 2^-127: what would need a smaller one is left out
        words[k] = scale >= 4u * k ? lo | (hi << 16) : 0u;
        if (k + 1 < PIECES) {
            const float2 a = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)lo, __NV_E4M3)));
            const float2 b = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)hi, __NV_E4M3)));
            f[0] = (f[0] - a.x) * 16.0f;
            f[1] = (f[1] - a.y) * 16.0f;
            f[2] = (f[2] - b.x) * 16.0f;
            f[3] = (f[3] - b.y) * 16.0f;
        }
    }
}

// What a block does after the routing: its share of gate and up (UP) or of down.  HALF: activations of gate and up are FP16.
template <bool UP, bool HALF, int PIECES, typename Finish>
__device__ __forceinline__ void stream_weights(const MoeParams& P, const MoeMaps& maps, MoeShared& S, uint32_t base, uint32_t blocks, Finish finish)
{
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t cols = UP ? P.hidden : P.inter, rows = UP ? P.inter : P.hidden;
    const uint32_t steps = (cols + 127) >> 7;
    const Waiter wait{P.spin_limit, &S.failed};
    Tiles<UP> tiles(S.R, rows, blockIdx.x, blocks);
    Tile t;
    uint32_t n = 0;                              // steps so far
    const uint32_t tmem = S.tmem;

    if (warp == 0) {
        if (lane == 0) {
            bool ok = true;
            while (ok && tiles.next(t)) {
                const uint32_t row0 = t.expert * (UP ? 2 * P.inter : P.hidden) + t.group * 8;
                for (uint32_t k = 0; k < steps; ++k, ++n) {
                    const uint32_t st = n % kMoeStages;
                    if (n >= kMoeStages && !(ok = wait(smem_u32(&S.empty[st]), (n / kMoeStages - 1) & 1))) break;
                    const uint32_t bar = smem_u32(&S.full[st]), to = base + st * kMoeStageBytes;
                    bar_expect(bar, t.groups * (UP ? 2048 : 1024));
                    if (P.skip_copy) continue;
                    // as few copies as there are bits in the number of groups: one of 8 rows takes the copy engine as long as one of 64
                    uint32_t i = 0;
#pragma unroll
                    for (int b = UP ? 3 : 4; b >= 0; --b) {
                        if (!(t.groups >> b & 1)) continue;
                        tensor_copy<1>(to + i * 1024, &maps.of[b], (int)(k * 128), (int)(row0 + 8 * i), bar);
                        if (UP) tensor_copy<1>(to + 8192 + i * 1024, &maps.of[b], (int)(k * 128), (int)(row0 + P.inter + 8 * i), bar);
                        i += 1u << b;
                    }
                }
            }
            // after a wait that gave up, copies may still be on their way into this block's shared memory
            if (!ok && !P.skip_copy)
                for (uint32_t i = n > kMoeStages ? n - kMoeStages : 0; i < n; ++i)
                    for (uint32_t q = 0; q <= P.spin_limit && !bar_try(smem_u32(&S.full[i % kMoeStages]), (i / kMoeStages) & 1); ++q) { }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            uint32_t tile = 0;
            bool ok = true;
            while (ok && tiles.next(t)) {
                const uint32_t buf = tile & 1, d = tmem + buf * 128;
                const uint32_t cols_d = (((t.count + 7) & ~7u) * PIECES + 15) & ~15u;      // what is behind the last piece is computed and not used
                const uint32_t idesc = P.idesc | ((cols_d >> 3) << 17);
                if (tile >= 2 && !(ok = wait(smem_u32(&S.acc_empty[buf]), ((tile >> 1) - 1) & 1))) break;
                tc_fence_after();
                for (uint32_t k = 0; k < steps; ++k, ++n) {
                    const uint32_t st = n % kMoeStages;
                    if (!(ok = wait(smem_u32(&S.full[st]), (n / kMoeStages) & 1))) break;
                    tc_fence_after();
                    const uint32_t at = base + st * kMoeStageBytes, sf = tmem + kMoeTmemScales + st * 8;
                    tmem_copy_scales(sf, at + 32768);
                    tmem_copy_scales(sf + 4, at + 32768 + 512);
                    const uint64_t da = operand_desc(at), db = operand_desc(at + 16384);
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j) mma_scaled<1>(d, da + 2 * j, db + 2 * j, idesc, sf, sf + 4, k | j);
                    mma_commit<1>(smem_u32(&S.empty[st]));
                }
                mma_commit<1>(smem_u32(&S.acc_full[buf]));
                ++tile;
            }
        }
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
                for (uint32_t q = 0; q < 4 && k + q < steps; ++q, ++n) {
                    const uint32_t st = n % kMoeStages;
                    if (!(ok = __all_sync(0xFFFFFFFFu, n < kMoeStages || wait(smem_u32(&S.empty[st]), (n / kMoeStages - 1) & 1)))) break;
                    const uint32_t at = base + st * kMoeStageBytes + 32768 + lane * 16;
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
        // a warp has a stage of its own: the time of all stages for the latency of its loads, and it sees every phase of its
        // stage's barrier (a wait by parity that skipped one would take the phase before for it)
        const uint32_t st = warp - 8, at = base + st * kMoeStageBytes;
        bool ok = true;
        while (ok && tiles.next(t)) {
            const uint32_t padded = (t.count + 7) & ~7u;
            for (uint32_t k = 0; k < steps; ++k, ++n) {
                if (n % kMoeStages != st) continue;
                const uint32_t col = k * 128 + lane * 4;
                for (uint32_t c = 0; c < padded; c += 8) {
                    uint4 raw[8];
#pragma unroll
                    for (uint32_t i = 0; i < 8; ++i) {
                        raw[i] = zero4();
                        if (c + i < t.count && col < cols) {
                            if (UP) {
                                const uint2 v = __ldg(reinterpret_cast<const uint2*>(P.x + 2 * ((uint64_t)S.row_token[t.row + c + i] * P.ld_x + col)));
                                raw[i].x = v.x;
                                raw[i].y = v.y;
                            } else {
                                raw[i] = *reinterpret_cast<const uint4*>(P.h + (uint64_t)(t.row + c + i) * P.inter_pad + col);
                            }
                        }
                    }
                    if (c == 0 && !(ok = __all_sync(0xFFFFFFFFu, n < kMoeStages || wait(smem_u32(&S.empty[st]), (n / kMoeStages - 1) & 1)))) break;
                    // four tokens at a time, whether they are there or not (their rows are): the chain of roundings is long
#pragma unroll
                    for (uint32_t f = 0; f < 8; f += 4) {
                        if (c + f >= t.count) break;
#pragma unroll
                        for (uint32_t i = f; i < f + 4; ++i) {
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
#pragma unroll
                            for (uint32_t q = 0; q < 4; ++q) v[q] = col + q < cols ? v[q] : 0.0f;
                            uint32_t words[PIECES], scale;
                            make_pieces<PIECES>(v, words, scale);
#pragma unroll
                            for (uint32_t q = 0; q < PIECES; ++q) {
                                const uint32_t r = q * padded + c + i;
                                sts32(at + 16384 + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4, words[q]);
                                if (lane == q) sts32(at + 32768 + 512 + (r & 31) * 16 + (r >> 5) * 4, scale >= 4u * q ? scale - 4u * q : 0u);
                            }
                        }
                    }
                }
                if (!ok) break;
                fence_async_shared();
                __syncwarp();
                if (lane == 0) bar_arrive(smem_u32(&S.full[st]));
            }
        }
    } else if (warp >= 4) {
        const uint32_t quad = warp & 3;
        uint32_t tile = 0;
        while (tiles.next(t)) {
            const uint32_t buf = tile & 1, padded = (t.count + 7) & ~7u;
            // the four warps go on, or stop, together: they meet at a barrier of their own
            uint32_t ok = wait(smem_u32(&S.acc_full[buf]), (tile >> 1) & 1) && !*wait.failed;
            asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %0, 0;\n\tbarrier.cta.red.and.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "+r"(ok) :: "memory");
            if (!ok) break;
            tc_fence_after();
            const uint32_t d = tmem + (quad * 32u << 16) + buf * 128;
            for (uint32_t c = 0; c < t.count; c += 8) {
                float part[PIECES][8];
#pragma unroll
                for (uint32_t q = 0; q < PIECES; ++q) tmem_ld8(d + q * padded + c, part[q]);
                tmem_ld_wait();
                // the smallest pieces first
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float sum = part[PIECES - 1][i];
#pragma unroll
                    for (int q = PIECES - 2; q >= 0; --q) sum += part[q][i];
                    part[0][i] = sum;
                }
                finish.store(t, c, quad, lane, part[0]);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_u32(&S.acc_empty[buf]));
            finish.tile_done(t);
            ++tile;
        }
    }
    __syncwarp();
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

// This block's part of the logits, logits[expert][token]: of the columns' parts of 128 the cluster's blocks take a share each, so
// that a cluster reads router and tokens once.  Products of a part are summed by the matrix instructions in FP32, the parts in FP64:
// what separates two experts' logits decides which weights are used, and 2^-24 of the sum of a part is far below what the
// activations' own rounding moves.
template <bool HALF>
__device__ __forceinline__ void router_logits(const MoeParams& P, uint32_t rank, MoeRouting& S)
{
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const uint32_t mt = (P.experts + 15) >> 4, nt = (P.tokens + 7) >> 3, tasks = mt * nt;
    const uint32_t all = (P.hidden + 127) >> 7, lo = all * rank / kMoeCluster, parts = all * (rank + 1) / kMoeCluster - lo;
    uint32_t split = 1;
    while (split * 2 * tasks <= kMoeWarps && split * 2 <= parts) split *= 2;
    for (uint32_t item = warp; item < tasks * split; item += kMoeWarps) {
        const uint32_t task = item / split, slice = item % split;
        const uint32_t e0 = (task / nt) * 16, tok = (task % nt) * 8 + g;
        const bool ok_a = e0 + g < P.experts, ok_b = e0 + g + 8 < P.experts, ok_x = tok < P.tokens;
        const uint8_t* ra = P.router + 2 * (uint64_t)(ok_a ? e0 + g : 0) * P.ld_router;
        const uint8_t* rb = P.router + 2 * (uint64_t)(ok_b ? e0 + g + 8 : 0) * P.ld_router;
        const uint8_t* xr = P.x + 2 * (uint64_t)(ok_x ? tok : 0) * P.ld_x;
        double sum[4] = {0, 0, 0, 0};
        for (uint32_t part = lo + parts * slice / split; part < lo + parts * (slice + 1) / split; ++part) {
            uint4 a[4], b[4], x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t col = part * 128 + j * 32 + 8 * t;
                const bool in = col < P.hidden;
                a[j] = in && ok_a ? ld_cached_v4(ra + 2 * col) : zero4();
                b[j] = in && ok_b ? ld_cached_v4(rb + 2 * col) : zero4();
                x[j] = in && ok_x ? ld_cached_v4(xr + 2 * col) : zero4();
                if (in && col + 8 > P.hidden) {
                    const uint32_t have = 2 * (P.hidden - col);
                    a[j] = first_bytes(a[j], have);
                    b[j] = first_bytes(b[j], have);
                    x[j] = first_bytes(x[j], have);
                }
            }
            float v[4] = {0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t first[4] = {a[j].x, b[j].x, a[j].y, b[j].y}, second[4] = {a[j].z, b[j].z, a[j].w, b[j].w};
                mma16<HALF>(v, first, x[j].x, x[j].y);
                mma16<HALF>(v, second, x[j].z, x[j].w);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) sum[q] += (double)v[q];
        }
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q) {
            const uint32_t e = e0 + g + 8 * (q >> 1), k = (task % nt) * 8 + 2 * t + (q & 1);
            if (split > 1) S.items[item * 128 + q * 32 + lane] = sum[q];
            else if (e < P.experts && k < P.tokens) S.logits[e * kMaxTokens + k] = sum[q];
        }
    }
    if (split == 1) return;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < tasks * 128; i += kMoeThreads) {
        const uint32_t task = i >> 7, q = (i >> 5) & 3, l = i & 31;
        double s = 0;
        for (uint32_t k = 0; k < split; ++k) s += S.items[(task * split + k) * 128 + q * 32 + l];
        const uint32_t e = (task / nt) * 16 + (l >> 2) + 8 * (q >> 1), tok = (task % nt) * 8 + 2 * (l & 3) + (q & 1);
        if (e < P.experts && tok < P.tokens) S.logits[e * kMaxTokens + tok] = s;
    }
}

// The top_k experts and their weights for this block's share of the tokens (rank, rank + 4, ...), one warp a token.
__device__ __forceinline__ void choose(const MoeParams& P, uint32_t rank, MoeRouting& S)
{
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t base = smem_u32(S.logits);
    for (uint32_t i = warp; rank + i * kMoeCluster < P.tokens; i += kMoeWarps) {
        const uint32_t tok = rank + i * kMoeCluster;
        unsigned long long key[kMaxExperts / 32];
#pragma unroll
        for (uint32_t k = 0; k < kMaxExperts / 32; ++k) {
            const uint32_t e = k * 32 + lane;
            key[k] = 0;
            if (e < P.experts) {
                double v = 0;
#pragma unroll
                for (uint32_t r = 0; r < kMoeCluster; ++r) v += ld_cluster_f64(map_shared(base + 8 * (e * kMaxTokens + tok), r));
                key[k] = order_key(v);
            }
        }
        double largest = 0;
        float total = 0;
        for (uint32_t j = 0; j < P.top_k; ++j) {
            unsigned long long best = 0;
            uint32_t where = 0;
#pragma unroll
            for (uint32_t k = 0; k < kMaxExperts / 32; ++k)
                if (key[k] > best) { best = key[k]; where = k; }
            const uint32_t hi = __reduce_max_sync(0xFFFFFFFFu, (uint32_t)(best >> 32));
            const uint32_t lo = __reduce_max_sync(0xFFFFFFFFu, (uint32_t)(best >> 32) == hi ? (uint32_t)best : 0u);
            const bool tie = (uint32_t)(best >> 32) == hi && (uint32_t)best == lo;
            const uint32_t e = __reduce_min_sync(0xFFFFFFFFu, tie ? where * 32 + lane : 0xFFFFFFFFu);
#pragma unroll
            for (uint32_t k = 0; k < kMaxExperts / 32; ++k)
                if (k * 32 + lane == e) key[k] = 0;
            const double v = value_of(((unsigned long long)hi << 32) | lo);
            if (j == 0) largest = v;
            const float p = expf((float)(v - largest));      // the difference in FP64, the exponential in FP32
            total += p;
            if (lane == 0) {
                S.id[i * P.top_k + j] = (uint16_t)e;
                S.p[i * P.top_k + j] = p;
            }
        }
        if (lane == 0)
            for (uint32_t j = 0; j < P.top_k; ++j) S.p[i * P.top_k + j] /= total;
    }
}

// From the tokens' choices to the experts' lists: tokens of an expert in ascending order, experts in ascending order.
__device__ __forceinline__ void make_lists(const MoeParams& P, MoeRouting& S, Routing& R)
{
    const uint32_t tid = threadIdx.x, n = P.tokens * P.top_k;
    for (uint32_t e = tid; e < kMaxExperts; e += kMoeThreads) S.mask[e] = 0;
    __syncthreads();
    for (uint32_t i = tid; i < n; i += kMoeThreads) atomicOr(&S.mask[S.id_all[i]], 1ull << (i / P.top_k));
    __syncthreads();
    if (tid < 32) {
        // each lane eight experts: counts of tokens, of chosen experts, of passes; sums over the lanes before
        uint32_t tokens = 0, active = 0, passes = 0;
        for (uint32_t k = 0; k < 8; ++k) {
            const uint32_t c = __popcll(S.mask[tid * 8 + k]);
            tokens += c;
            active += c != 0;
            passes += (c + kMoePass - 1) / kMoePass;
        }
        uint32_t a = tokens, b = active, c = passes;
        for (uint32_t d = 1; d < 32; d <<= 1) {
            const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, a, d), y = __shfl_up_sync(0xFFFFFFFFu, b, d), z = __shfl_up_sync(0xFFFFFFFFu, c, d);
            if (tid >= d) { a += x; b += y; c += z; }
        }
        uint32_t row = a - tokens, at = b - active, pass = c - passes;
        for (uint32_t k = 0; k < 8; ++k) {
            const uint32_t cnt = __popcll(S.mask[tid * 8 + k]);
            if (!cnt) continue;
            R.expert[at] = (uint16_t)(tid * 8 + k);
            R.first[at] = (uint16_t)row;
            R.pass[at] = (uint16_t)pass;
            ++at;
            row += cnt;
            pass += (cnt + kMoePass - 1) / kMoePass;
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

struct RowFinder {
    const MoeRouting& S;
    const Routing& R;
    // row of a token in the list of expert e: the first row of e is that of the number of (token, expert) pairs before it
    __device__ __forceinline__ uint32_t operator()(uint32_t e, uint32_t token) const
    {
        uint32_t lo = 0, hi = R.n_active;
        while (hi - lo > 1) {
            const uint32_t mid = (lo + hi) / 2;
            if (R.expert[mid] <= e) lo = mid; else hi = mid;
        }
        return R.first[lo] + __popcll(S.mask[e] & ((1ull << token) - 1));
    }
};

// Barriers and tensor memory; all threads.
__device__ __forceinline__ void moe_setup(MoeShared& S)
{
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (warp == 0 && lane == 0) {
        for (uint32_t i = 0; i < kMoeStages; ++i) { bar_init(smem_u32(&S.full[i]), 3); bar_init(smem_u32(&S.empty[i]), 1); }
        for (uint32_t i = 0; i < 2; ++i) { bar_init(smem_u32(&S.acc_full[i]), 1); bar_init(smem_u32(&S.acc_empty[i]), 4); }
        S.failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
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
    __device__ __forceinline__ void store(const Tile& t, uint32_t c, uint32_t quad, uint32_t lane, const float v[8]) const
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
    __device__ __forceinline__ void store(const Tile& t, uint32_t c, uint32_t quad, uint32_t lane, const float v[8]) const
    {
        const uint32_t row = quad * 32 + lane, r = t.group * 8 + row;
        if (row >= t.groups * 8 || r >= P.hidden) return;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (c + i < t.count) P.z[(uint64_t)(t.row + c + i) * P.hidden_pad + r] = v[i];
    }
    // the four warps: whoever completes a group's last pass adds the experts up, four columns of a token a thread
    __device__ __forceinline__ void tile_done(const Tile& t) const
    {
        const uint32_t tid = threadIdx.x & 127;
        __threadfence();
        asm volatile("bar.sync 1, 128;" ::: "memory");
        if (tid < t.groups) {
            S.last[tid] = atomicAdd(&P.done[t.group + tid], 1u) + 1 == n_passes;
            __threadfence();
        }
        asm volatile("bar.sync 1, 128;" ::: "memory");
        const uint32_t g = (tid & 31) >> 1, r = (t.group + g) * 8 + (tid & 1) * 4;
        if (g < t.groups && S.last[g] && r < P.hidden) {
            for (uint32_t tok = tid >> 5; tok < P.tokens; tok += 4) {
                float y[4] = {0, 0, 0, 0};
                const uint16_t* rows = S.row_of + tok * P.top_k;
#pragma unroll 8
                for (uint32_t j = 0; j < P.top_k; ++j) {
                    const float4 z = __ldcg(reinterpret_cast<const float4*>(P.z + (uint64_t)rows[j] * P.hidden_pad + r));
                    y[0] += z.x; y[1] += z.y; y[2] += z.z; y[3] += z.w;
                }
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) {
                    if (r + i >= P.hidden) break;
                    if (HALF) reinterpret_cast<__half*>(P.y)[(uint64_t)tok * P.ld_y + r + i] = __float2half_rn(y[i]);
                    else reinterpret_cast<__nv_bfloat16*>(P.y)[(uint64_t)tok * P.ld_y + r + i] = __float2bfloat16_rn(y[i]);
                }
            }
        }
        asm volatile("bar.sync 1, 128;" ::: "memory");
    }
};

// hidden vectors: twelve bits in three pieces err a sixteenth of what rounding y to BF16 does; FP16 takes sixteen in four
template <bool HALF> constexpr int kHiddenPieces = HALF ? 4 : 3;

template <bool HALF>
__global__ void __launch_bounds__(kMoeThreads, 1)
moe_up_kernel(const __grid_constant__ MoeMaps maps, const __grid_constant__ MoeParams P)
{
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    uint8_t* aligned = raw + (base - smem_u32(raw));
    MoeShared& S = *reinterpret_cast<MoeShared*>(aligned + kMoeStages * kMoeStageBytes);
    MoeRouting& T = *reinterpret_cast<MoeRouting*>(aligned);
    const uint32_t tid = threadIdx.x, rank = cluster_rank();
    const uint32_t n_rows = P.tokens * P.top_k;

    grid_launch_dependents();
    if (tid < kMoeHeights) prefetch_map(&maps.of[tid]);
    moe_setup(S);
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
    const RowFinder row_of{T, S.R};
    for (uint32_t i = tid; i < n_rows; i += kMoeThreads) {
        const uint32_t r = row_of(T.id_all[i], i / P.top_k);
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
    stream_weights<true, HALF, 3>(P, maps, S, base, gridDim.x, FinishUp{P, S});
    __syncthreads();
    if (tid < 64 && tid >= 32) tmem_free<1>(S.tmem, kMoeTmemCols);
}

template <bool HALF>
__global__ void __launch_bounds__(kMoeThreads, 1)
moe_down_kernel(const __grid_constant__ MoeMaps maps, const __grid_constant__ MoeParams P)
{
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    MoeShared& S = *reinterpret_cast<MoeShared*>(raw + (base - smem_u32(raw)) + kMoeStages * kMoeStageBytes);
    const uint32_t tid = threadIdx.x;
    if (tid < kMoeHeights) prefetch_map(&maps.of[tid]);
    moe_setup(S);
    grid_wait();
    const uint32_t n_active = P.route[0], n_passes = P.route[1];
    for (uint32_t i = tid; i <= n_active; i += kMoeThreads) {
        if (i < n_active) S.R.expert[i] = (uint16_t)P.route[2 + i];
        const uint32_t v = P.route[2 + kMaxExperts + i];
        S.R.first[i] = (uint16_t)v;
        S.R.pass[i] = (uint16_t)(v >> 16);
    }
    for (uint32_t i = tid; i < P.tokens * P.top_k; i += kMoeThreads) S.row_of[i] = (uint16_t)P.row_of[i];
    if (tid == 0) { S.R.n_active = n_active; S.R.n_passes = n_passes; }
    __syncthreads();
    stream_weights<false, HALF, kHiddenPieces<HALF>>(P, maps, S, base, gridDim.x, FinishDown<HALF>{P, S, n_passes});
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
    if (!up_blocks) return cudaErrorUnknown;
    cudaLaunchConfig_t cfg{};
    cfg.blockDim = dim3(kMoeThreads);
    cfg.dynamicSmemBytes = kMoeSmem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    cfg.attrs = at;
    cfg.numAttrs = 1;
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {kMoeCluster, 1, 1};
    cfg.gridDim = dim3(up_blocks);
    e = cudaLaunchKernelEx(&cfg, moe_up_kernel<HALF>, up, P);
    if (e != cudaSuccess) return e;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((uint32_t)sm_count());
    return cudaLaunchKernelEx(&cfg, moe_down_kernel<HALF>, down, P);
}

zc_status moe_read_timeout(cudaStream_t st) { return read_timeout(st); }

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
    P.spin_limit = test_knobs().spin_limit;
    P.skip_copy = test_knobs().skip_copy;
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
