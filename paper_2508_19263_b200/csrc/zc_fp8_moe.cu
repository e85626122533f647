// zc_fp8_moe: a mixture-of-experts layer for a few tokens, in two kernels.
//
// With a few tokens the time goes into reading the chosen experts' weights once, so both kernels stream them straight into
// registers: a warp's step is a tile of 16 rows x 64 bytes (two 16-byte loads a lane, four steps ahead), turned into BF16 (FP16
// for FP16 activations), which hold FP8 values exactly, and multiplied with up to 32 tokens by warp-wide matrix
// instructions.  The order of k inside an instruction is free as long as both operands agree on it: lane 4 g + t takes bytes
// 16 t .. 16 t + 15 of rows g and g + 8, so no weight passes through shared memory.  Tiles of all chosen experts form one
// sequence that is cut into equal ranges, one per block; within a block every warp takes its share of k of each tile, and the
// warps' parts are added up in shared memory in the order of the warps.
//
//   kernel 1  routes (every cluster for itself, so that no block waits for another cluster), then gate and up: a tile is 8 rows of
//             gate and the same 8 of up, so that a thread ends with both and writes silu(gate) * up * p
//   kernel 2  down: 16 rows a tile, one FP32 row of partial results per (token, expert); the block that completes a
//             tile's last expert adds the experts up in the order of the token's list
#include "zc_fp8.cuh"

namespace zc {

constexpr uint32_t kMoeWarps = 8, kMoeThreads = 32 * kMoeWarps;
constexpr uint32_t kMoeCluster = 4;
constexpr uint32_t kMoeSlots = 8;                // results of 16 rows x 8 tokens that a block adds up at a time
constexpr uint32_t kMoePass = 32;                // tokens that share a reading of a tile
constexpr uint32_t kMoeAhead = 4;                // steps that a warp's loads are ahead
constexpr uint32_t kMaxTokens = ZC_FP8_MOE_MAX_TOKENS, kMaxExperts = ZC_FP8_MOE_MAX_EXPERTS;
constexpr uint32_t kMaxRows = kMaxTokens * ZC_FP8_MOE_MAX_TOP_K;

struct MoeParams {
    const uint8_t *x, *router;                   // rows of BF16 or FP16
    uint64_t ld_x, ld_router;                    // elements
    const uint8_t *gate_up, *gate_up_scales, *down, *down_scales;
    uint64_t ld_gate_up, ld_down;
    uint32_t tokens, experts, top_k, hidden, inter;
    uint32_t hidden_pad, inter_pad;              // rounded up to 64 columns
    uint32_t *ids_out;
    float *weights_out;
    uint8_t *y;
    uint64_t ld_y;                               // elements
    // workspace
    uint32_t *route;                             // [0]: chosen experts; then their numbers, their first rows
    uint32_t *row_of;                            // [tokens][top_k]: row of a token's j-th expert
    uint32_t *done;                              // [tiles of down]: experts whose part is written
    uint16_t *h;                                 // [rows][2][inter_pad]: BF16, upper and lower part
    float *z;                                    // [rows][hidden_pad]
};

// What a block knows of the routing.
struct Routing {
    uint32_t n_active, n_passes;                 // chosen experts; of up to 32 tokens each
    uint16_t expert[kMaxExperts];
    uint16_t first[kMaxExperts + 1];             // first row of an expert's tokens
    uint16_t pass[kMaxExperts + 1];              // passes of the experts before
};
struct SlotInfo { uint16_t active, count; uint32_t tile, row; };
struct MoeShared {
    Routing R;
    SlotInfo slot[2][kMoeSlots];
    float row_p[kMaxRows];
    uint8_t row_token[kMaxRows];
    float p[kMaxRows];                           // [tokens of this block][top_k] of the cluster's share, then of all tokens
    uint16_t id[kMaxRows];
    float p_all[kMaxRows];
    uint16_t id_all[kMaxRows];
    unsigned long long mask[kMaxExperts];        // tokens that chose the expert
    uint32_t last[kMoeSlots];
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// two FP8 bytes as a pair of FP16 or BF16 (both exact)
template <bool E5M2, bool HALF>
__device__ __forceinline__ uint32_t widen(uint32_t two)
{
    const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, E5M2 ? __NV_E5M2 : __NV_E4M3);
    if (HALF) return (uint32_t)r.x | ((uint32_t)r.y << 16);
    const float2 f = __half22float2(__half2(r));
    return pack_bf16(f.x, f.y);
}
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

// Where a warp's loads, or its products, are: expert, tile of rows, pass over the expert's tokens, chunk of 64 columns.
struct Cursor {
    uint32_t active, tile, pass, chunk;
};

// UP: tiles of 8 + 8 rows of gate and up, x as the other operand; else tiles of 16 rows of down, h as the other operand.
template <bool UP, bool E5M2, bool HALF>
struct Stream {
    const MoeParams& P;
    MoeShared& S;
    float4* parts;                               // [2][kMoeSlots][kMoeWarps][32]
    uint32_t tiles, cols, c_lo, c_hi, n_warps;
    uint32_t g, t, lane, warp;

    struct Step { uint4 a, b; uint32_t s; };

    __device__ __forceinline__ uint32_t passes(uint32_t active) const { return S.R.pass[active + 1] - S.R.pass[active]; }

    __device__ __forceinline__ void advance(Cursor& c) const
    {
        if (++c.chunk < c_hi) return;
        c.chunk = c_lo;
        if (++c.pass < passes(c.active)) return;
        c.pass = 0;
        if (++c.tile < tiles) return;
        c.tile = 0;
        ++c.active;
    }

    __device__ __forceinline__ Step load(const Cursor& c) const
    {
        Step r{zero4(), zero4(), 0};
        const uint32_t e = S.R.expert[c.active], col = c.chunk * 64 + 16 * t, sc = c.chunk >> 1;
        const uint32_t limit = UP ? P.inter : P.hidden;
        const uint32_t row_a = UP ? c.tile * 8 + g : c.tile * 16 + g, row_b = UP ? row_a : row_a + 8;
        const uint64_t ld = UP ? P.ld_gate_up : P.ld_down;
        const uint8_t* w = UP ? P.gate_up + (uint64_t)e * 2 * P.inter * ld : P.down + (uint64_t)e * P.hidden * ld;
        const uint32_t sld = (cols + 127) >> 7, srows = (limit + 127) >> 7;
        const uint8_t* s = (UP ? P.gate_up_scales + (uint64_t)e * 2 * srows * sld : P.down_scales + (uint64_t)e * srows * sld) + sc;
        if (col < cols) {
            if (row_a < limit) r.a = ld_stream_v4(w + (uint64_t)row_a * ld + col);
            if (row_b < limit) r.b = ld_stream_v4(w + (uint64_t)(UP ? P.inter + row_b : row_b) * ld + col);
        }
        const uint32_t srow = (UP ? c.tile * 8 : c.tile * 16) >> 7;
        if (srow < srows) {
            const uint32_t s0 = __ldg(s + (uint64_t)srow * sld), s1 = UP ? __ldg(s + (uint64_t)(srows + srow) * sld) : s0;
            r.s = s0 | (s1 << 8);
        }
        return r;
    }

    __device__ __forceinline__ void multiply(const Cursor& c, Step w, float acc[4][4], uint32_t row, uint32_t count) const
    {
        const uint32_t col = c.chunk * 64 + 16 * t;
        if (col + 16 > cols) {
            const uint32_t n = col < cols ? cols - col : 0;
            w.a = first_bytes(w.a, n);
            w.b = first_bytes(w.b, n);
        }
        const uint32_t wa[4] = {w.a.x, w.a.y, w.a.z, w.a.w}, wb[4] = {w.b.x, w.b.y, w.b.z, w.b.w};
        uint32_t a[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            a[j][0] = widen<E5M2, HALF>(wa[j] & 0xFFFFu);
            a[j][1] = widen<E5M2, HALF>(wb[j] & 0xFFFFu);
            a[j][2] = widen<E5M2, HALF>(wa[j] >> 16);
            a[j][3] = widen<E5M2, HALF>(wb[j] >> 16);
        }
        const float s0 = scale_value(w.s & 255u), s1 = UP ? scale_value(w.s >> 8) : s0;
#pragma unroll
        for (uint32_t n = 0; n < 4; ++n) {
            if (n * 8 >= count) break;
            float v[4] = {0, 0, 0, 0};
            const bool mine = n * 8 + g < count;
            if (UP) {
                const uint8_t* x = P.x + 2 * ((uint64_t)(mine ? S.row_token[row + n * 8 + g] : 0) * P.ld_x + col);
                uint4 lo = mine && col < cols ? ld_cached_v4(x) : zero4();
                uint4 hi = mine && col + 8 < cols ? ld_cached_v4(x + 16) : zero4();
                if (col + 16 > cols) {
                    const uint32_t have = col < cols ? 2 * (cols - col) : 0;
                    lo = first_bytes(lo, have);
                    hi = first_bytes(hi, have > 16 ? have - 16 : 0);
                }
                mma16<HALF>(v, a[0], lo.x, lo.y);
                mma16<HALF>(v, a[1], lo.z, lo.w);
                mma16<HALF>(v, a[2], hi.x, hi.y);
                mma16<HALF>(v, a[3], hi.z, hi.w);
            } else {
                // written by the kernel before this one: through L2, not the read-only path that it might have been fetched by
                const uint16_t* h = P.h + (uint64_t)(row + n * 8 + (mine ? g : 0)) * 2 * P.inter_pad + col;
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    const uint4* q = reinterpret_cast<const uint4*>(h + part * P.inter_pad);
                    const uint4 lo = mine ? q[0] : zero4(), hi = mine ? q[1] : zero4();
                    mma16<false>(v, a[0], lo.x, lo.y);
                    mma16<false>(v, a[1], lo.z, lo.w);
                    mma16<false>(v, a[2], hi.x, hi.y);
                    mma16<false>(v, a[3], hi.z, hi.w);
                }
            }
            acc[n][0] = fmaf(v[0], s0, acc[n][0]);
            acc[n][1] = fmaf(v[1], s0, acc[n][1]);
            acc[n][2] = fmaf(v[2], s1, acc[n][2]);
            acc[n][3] = fmaf(v[3], s1, acc[n][3]);
        }
    }

    // All warps, for the block's range of the tiles; `finish(batch)` after each batch of up to kMoeSlots results.
    template <typename Finish>
    __device__ __forceinline__ void run(uint32_t first, uint32_t end, Finish finish)
    {
        if (first >= end) return;
        const uint32_t chunks = (cols + 63) >> 6;
        n_warps = chunks < kMoeWarps ? chunks : kMoeWarps;
        const bool busy = warp < n_warps;
        c_lo = busy ? chunks * warp / n_warps : 0;
        c_hi = busy ? chunks * (warp + 1) / n_warps : 1;
        // the tile numbered `first`: passes over an expert's tokens lie next to each other, so that the second finds the tile cached
        Cursor at{0, 0, 0, c_lo};
        while (first >= (uint32_t)S.R.pass[at.active + 1] * tiles) ++at.active;
        const uint32_t rest = first - S.R.pass[at.active] * tiles;
        at.tile = rest / passes(at.active);
        at.pass = rest % passes(at.active);
        Cursor ahead = at;
        uint32_t to_load = busy ? (end - first) * (c_hi - c_lo) : 0;
        Step ring[kMoeAhead];
#pragma unroll
        for (uint32_t i = 0; i < kMoeAhead; ++i) {
            ring[i] = Step{zero4(), zero4(), 0};
            if (to_load) { ring[i] = load(ahead); advance(ahead); --to_load; }
        }
        float acc[4][4] = {};
        uint32_t batch = 0, used = 0, left = end - first;
        while (left) {
#pragma unroll
            for (uint32_t i = 0; i < kMoeAhead; ++i) {
                if (!left) break;
                const uint32_t row = S.R.first[at.active] + at.pass * kMoePass;
                const uint32_t n = S.R.first[at.active + 1] - row, count = n < kMoePass ? n : kMoePass, need = (count + 7) >> 3;
                if (used + need > kMoeSlots) {               // uniform: every warp sees the same tiles
                    finish(batch, used);
                    ++batch;
                    used = 0;
                }
                if (busy) {
                    multiply(at, ring[i], acc, row, count);
                    if (to_load) { ring[i] = load(ahead); advance(ahead); --to_load; }
                }
                if (!busy || at.chunk + 1 == c_hi) {
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k) {
                        if (k >= need) break;
                        if (busy) parts[(((batch & 1) * kMoeSlots + used + k) * kMoeWarps + warp) * 32 + lane] = make_float4(acc[k][0], acc[k][1], acc[k][2], acc[k][3]);
                        if (warp == 0 && lane == 0)
                            S.slot[batch & 1][used + k] = SlotInfo{(uint16_t)at.active, (uint16_t)(count - 8 * k < 8 ? count - 8 * k : 8), at.tile, row + 8 * k};
#pragma unroll
                        for (int q = 0; q < 4; ++q) acc[k][q] = 0.0f;
                    }
                    used += need;
                    --left;
                }
                advance(at);
            }
        }
        finish(batch, used);
    }

    __device__ __forceinline__ float4 sum(uint32_t batch, uint32_t slot) const
    {
        float4 s = make_float4(0, 0, 0, 0);
        for (uint32_t w = 0; w < n_warps; ++w) {
            const float4 v = parts[(((batch & 1) * kMoeSlots + slot) * kMoeWarps + w) * 32 + lane];
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        return s;
    }
};

// ---- routing ----------------------------------------------------------------------------------------------------------

// order of doubles as unsigned numbers; NaN below everything, both zeros alike
__device__ __forceinline__ unsigned long long order_key(double v)
{
    if (v != v) return 0;
    const unsigned long long b = (unsigned long long)__double_as_longlong(v + 0.0);
    return (b >> 63) ? ~b : b | (1ull << 63);
}
__device__ __forceinline__ double ld_cluster_f64(uint32_t addr)
{
    double v;
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(addr) : "memory");
    return v;
}

// The logits of this block's experts (tiles of 16: rank, rank + 4, ...) for all tokens, logits[local expert][token].  Products
// of parts of 128 columns are summed by the matrix instructions in FP32, the parts in FP64: what separates two experts' logits
// decides which weights are used, and 2^-24 of the sum of a part is far below what the activations' own rounding moves.
template <bool HALF>
__device__ __forceinline__ void router_logits(const MoeParams& P, uint32_t rank, double* items, double* logits)
{
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const uint32_t all_tiles = (P.experts + 15) >> 4, nt = (P.tokens + 7) >> 3;
    const uint32_t mt = all_tiles > rank ? (all_tiles - rank + kMoeCluster - 1) / kMoeCluster : 0, tasks = mt * nt;
    const uint32_t parts = (P.hidden + 127) >> 7;
    uint32_t split = 1;
    while (split * 2 * tasks <= kMoeWarps && split * 2 <= parts) split *= 2;
    for (uint32_t item = warp; item < tasks * split; item += kMoeWarps) {
        const uint32_t task = item / split, slice = item % split;
        const uint32_t e0 = (rank + (task / nt) * kMoeCluster) * 16, tok = (task % nt) * 8 + g;
        const bool ok_a = e0 + g < P.experts, ok_b = e0 + g + 8 < P.experts, ok_x = tok < P.tokens;
        const uint8_t* ra = P.router + 2 * (uint64_t)(ok_a ? e0 + g : 0) * P.ld_router;
        const uint8_t* rb = P.router + 2 * (uint64_t)(ok_b ? e0 + g + 8 : 0) * P.ld_router;
        const uint8_t* xr = P.x + 2 * (uint64_t)(ok_x ? tok : 0) * P.ld_x;
        double sum[4] = {0, 0, 0, 0};
        for (uint32_t part = parts * slice / split; part < parts * (slice + 1) / split; ++part) {
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
                const uint32_t lo[4] = {a[j].x, b[j].x, a[j].y, b[j].y}, hi[4] = {a[j].z, b[j].z, a[j].w, b[j].w};
                mma16<HALF>(v, lo, x[j].x, x[j].y);
                mma16<HALF>(v, hi, x[j].z, x[j].w);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) sum[q] += (double)v[q];
        }
        double* to = items + item * 128 + lane;
#pragma unroll
        for (int q = 0; q < 4; ++q) to[q * 32] = sum[q];
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < tasks * 128; i += kMoeThreads) {
        const uint32_t task = i >> 7, q = (i >> 5) & 3, l = i & 31;
        double s = 0;
        for (uint32_t k = 0; k < split; ++k) s += items[(task * split + k) * 128 + q * 32 + l];
        const uint32_t e = (task / nt) * 16 + (l >> 2) + 8 * (q >> 1), tok = (task % nt) * 8 + 2 * (l & 3) + (q & 1);
        if (tok < P.tokens) logits[e * kMaxTokens + tok] = s;
    }
}

// The top_k experts and their weights for this block's share of the tokens (rank, rank + 4, ...), one warp a token.
__device__ __forceinline__ void choose(const MoeParams& P, uint32_t rank, const double* logits, MoeShared& S)
{
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t base = smem_u32(logits);
    for (uint32_t i = warp; rank + i * kMoeCluster < P.tokens; i += kMoeWarps) {
        const uint32_t tok = rank + i * kMoeCluster;
        unsigned long long key[kMaxExperts / 32];
#pragma unroll
        for (uint32_t k = 0; k < kMaxExperts / 32; ++k) {
            const uint32_t e = k * 32 + lane;
            key[k] = 0;
            // + 1: an expert that is there beats a place behind the last one even when its logit is NaN
            if (e < P.experts) {
                const uint32_t tile = e >> 4, local = (tile / kMoeCluster) * 16 + (e & 15);
                const unsigned long long o = order_key(ld_cluster_f64(map_shared(base + 8 * (local * kMaxTokens + tok), tile % kMoeCluster)));
                key[k] = o ? o : 1;
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
            const uint32_t tile = e >> 4, local = (tile / kMoeCluster) * 16 + (e & 15);
            const double v = ld_cluster_f64(map_shared(base + 8 * (local * kMaxTokens + tok), tile % kMoeCluster));
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
__device__ __forceinline__ void make_lists(const MoeParams& P, MoeShared& S)
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
            S.R.expert[at] = (uint16_t)(tid * 8 + k);
            S.R.first[at] = (uint16_t)row;
            S.R.pass[at] = (uint16_t)pass;
            ++at;
            row += cnt;
            pass += (cnt + kMoePass - 1) / kMoePass;
        }
        if (tid == 31) {
            S.R.n_active = b;
            S.R.n_passes = c;
            S.R.first[b] = (uint16_t)a;
            S.R.pass[b] = (uint16_t)c;
        }
    }
    __syncthreads();
}

struct RowFinder {
    const MoeShared& S;
    // row of a token in the list of expert e: the first row of e is that of the number of (token, expert) pairs before it
    __device__ __forceinline__ uint32_t operator()(uint32_t e, uint32_t token) const
    {
        uint32_t lo = 0, hi = S.R.n_active;
        while (hi - lo > 1) {
            const uint32_t mid = (lo + hi) / 2;
            if (S.R.expert[mid] <= e) lo = mid; else hi = mid;
        }
        return S.R.first[lo] + __popcll(S.mask[e] & ((1ull << token) - 1));
    }
};

constexpr size_t kMoePartBytes = 2ull * kMoeSlots * kMoeWarps * 32 * sizeof(float4);          // 64 KiB
constexpr size_t kMoeSmem = kMoePartBytes + sizeof(MoeShared);
static_assert(kMoePartBytes >= (32 * 128 + 64 * kMaxTokens) * sizeof(double), "the router's sums lie where the tiles' parts will be");

template <bool E5M2, bool HALF>
__global__ void __launch_bounds__(kMoeThreads, 2)
moe_up_kernel(const __grid_constant__ MoeParams P)
{
    extern __shared__ __align__(16) uint8_t raw[];
    float4* parts = reinterpret_cast<float4*>(raw);
    MoeShared& S = *reinterpret_cast<MoeShared*>(raw + kMoePartBytes);
    double* items = reinterpret_cast<double*>(raw);
    double* logits = items + 32 * 128;
    const uint32_t tid = threadIdx.x, rank = cluster_rank();
    const uint32_t n_rows = P.tokens * P.top_k;

    grid_launch_dependents();
    router_logits<HALF>(P, rank, items, logits);
    cluster_sync();
    choose(P, rank, logits, S);
    cluster_sync();
    for (uint32_t i = tid; i < n_rows; i += kMoeThreads) {
        const uint32_t tok = i / P.top_k, j = i % P.top_k, at = (tok / kMoeCluster) * P.top_k + j, from = tok % kMoeCluster;
        float p;
        uint16_t id;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(p) : "r"(map_shared(smem_u32(&S.p[at]), from)) : "memory");
        asm volatile("ld.shared::cluster.u16 %0, [%1];" : "=h"(id) : "r"(map_shared(smem_u32(&S.id[at]), from)) : "memory");
        S.p_all[i] = p;
        S.id_all[i] = id;
    }
    cluster_sync();                              // nobody reads this block's shared memory any more
    make_lists(P, S);
    const RowFinder row_of{S};
    for (uint32_t i = tid; i < n_rows; i += kMoeThreads) {
        const uint32_t r = row_of(S.id_all[i], i / P.top_k);
        S.row_p[r] = S.p_all[i];
        S.row_token[r] = (uint8_t)(i / P.top_k);
        if (blockIdx.x == 0) {
            P.row_of[i] = r;
            if (P.ids_out) P.ids_out[i] = S.id_all[i];
            if (P.weights_out) P.weights_out[i] = S.p_all[i];
        }
    }
    if (blockIdx.x == 0) {
        for (uint32_t i = tid; i < (P.hidden + 15) / 16; i += kMoeThreads) P.done[i] = 0;
        for (uint32_t i = tid; i <= S.R.n_active; i += kMoeThreads) {
            if (i < S.R.n_active) P.route[2 + i] = S.R.expert[i];
            P.route[2 + kMaxExperts + i] = (uint32_t)S.R.first[i] | ((uint32_t)S.R.pass[i] << 16);
        }
        if (tid == 0) { P.route[0] = S.R.n_active; P.route[1] = S.R.n_passes; }
    }
    __syncthreads();

    const uint32_t tiles = P.inter_pad / 8;
    Stream<true, E5M2, HALF> W{P, S, parts, tiles, P.hidden, 0, 0, 0, (tid & 31) >> 2, tid & 3, tid & 31, tid >> 5};
    const uint64_t total = (uint64_t)tiles * S.R.n_passes;
    W.run((uint32_t)(total * blockIdx.x / gridDim.x), (uint32_t)(total * (blockIdx.x + 1) / gridDim.x), [&](uint32_t batch, uint32_t used) {
        __syncthreads();
        const uint32_t slot = tid >> 5;
        if (slot < used) {
            const SlotInfo I = S.slot[batch & 1][slot];
            const float4 v = W.sum(batch, slot);
            const uint32_t ch = I.tile * 8 + W.g;
#pragma unroll
            for (uint32_t k = 0; k < 2; ++k) {
                const uint32_t n = 2 * W.t + k;
                if (n >= I.count) continue;
                const float gate = k ? v.y : v.x, up = k ? v.w : v.z;
                const float h = gate / (1.0f + expf(-gate)) * up * S.row_p[I.row + n];
                // upper and lower half in BF16 each, 16 bits together: one of 8 bits would err as much as rounding y does
                const __nv_bfloat16 hi = __float2bfloat16_rn(h);
                const __nv_bfloat16 lo = __float2bfloat16_rn(isinf(__bfloat162float(hi)) ? 0.0f : h - __bfloat162float(hi));
                uint16_t* to = P.h + (uint64_t)(I.row + n) * 2 * P.inter_pad + ch;
                to[0] = *reinterpret_cast<const uint16_t*>(&hi);
                to[P.inter_pad] = *reinterpret_cast<const uint16_t*>(&lo);
            }
        }
    });
}

template <bool E5M2, bool HALF>
__global__ void __launch_bounds__(kMoeThreads, 2)
moe_down_kernel(const __grid_constant__ MoeParams P)
{
    extern __shared__ __align__(16) uint8_t raw[];
    float4* parts = reinterpret_cast<float4*>(raw);
    MoeShared& S = *reinterpret_cast<MoeShared*>(raw + kMoePartBytes);
    const uint32_t tid = threadIdx.x;
    grid_wait();
    const uint32_t n_active = P.route[0], n_passes = P.route[1];
    for (uint32_t i = tid; i <= n_active; i += kMoeThreads) {
        if (i < n_active) S.R.expert[i] = (uint16_t)P.route[2 + i];
        const uint32_t v = P.route[2 + kMaxExperts + i];
        S.R.first[i] = (uint16_t)v;
        S.R.pass[i] = (uint16_t)(v >> 16);
    }
    __syncthreads();
    const uint32_t tiles = (P.hidden + 15) / 16;
    Stream<false, E5M2, false> W{P, S, parts, tiles, P.inter, 0, 0, 0, (tid & 31) >> 2, tid & 3, tid & 31, tid >> 5};
    const uint64_t total = (uint64_t)tiles * n_passes;
    W.run((uint32_t)(total * blockIdx.x / gridDim.x), (uint32_t)(total * (blockIdx.x + 1) / gridDim.x), [&](uint32_t batch, uint32_t used) {
        __syncthreads();
        const uint32_t slot = tid >> 5;
        if (slot < used) {
            const SlotInfo I = S.slot[batch & 1][slot];
            const float4 v = W.sum(batch, slot);
            float* z = P.z + (uint64_t)(I.row + 2 * W.t) * P.hidden_pad + I.tile * 16 + W.g;
            if (2 * W.t < I.count) { z[0] = v.x; z[8] = v.z; }
            if (2 * W.t + 1 < I.count) { z[P.hidden_pad] = v.y; z[P.hidden_pad + 8] = v.w; }
            __threadfence();
        }
        __syncthreads();
        // one arrival per tile and pass: at its first slot
        if (tid < used) {
            const SlotInfo I = S.slot[batch & 1][tid];
            const uint32_t r = I.row - S.R.first[I.active];
            S.last[tid] = r % kMoePass == 0 ? atomicAdd(&P.done[I.tile], 1u) + 1 == n_passes : 0;
            __threadfence();
        }
        __syncthreads();
        for (uint32_t k = 0; k < used; ++k) {
            if (!S.last[k]) continue;
            const uint32_t row0 = S.slot[batch & 1][k].tile * 16;
            for (uint32_t i = tid; i < P.tokens * 16; i += kMoeThreads) {
                const uint32_t tok = i >> 4, r = row0 + (i & 15);
                if (r >= P.hidden) continue;
                float y = 0;
                for (uint32_t j = 0; j < P.top_k; ++j) y += __ldcg(P.z + (uint64_t)P.row_of[tok * P.top_k + j] * P.hidden_pad + r);
                if (HALF) reinterpret_cast<__half*>(P.y)[(uint64_t)tok * P.ld_y + r] = __float2half_rn(y);
                else reinterpret_cast<__nv_bfloat16*>(P.y)[(uint64_t)tok * P.ld_y + r] = __float2bfloat16_rn(y);
            }
        }
    });
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
    o.done = take(4 * (hidden_pad / 16));
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

template <bool E5M2, bool HALF>
static cudaError_t launch_moe(const MoeParams& P, cudaStream_t st)
{
    cudaError_t e = cudaFuncSetAttribute(moe_up_kernel<E5M2, HALF>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMoeSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(moe_down_kernel<E5M2, HALF>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMoeSmem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cfg.blockDim = dim3(kMoeThreads);
    cfg.dynamicSmemBytes = kMoeSmem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    cfg.attrs = at;
    cfg.numAttrs = 1;
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {kMoeCluster, 1, 1};
    cfg.gridDim = dim3(2 * (uint32_t)sm_count() / kMoeCluster * kMoeCluster);
    e = cudaLaunchKernelEx(&cfg, moe_up_kernel<E5M2, HALF>, P);
    if (e != cudaSuccess) return e;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(2 * (uint32_t)sm_count());
    return cudaLaunchKernelEx(&cfg, moe_down_kernel<E5M2, HALF>, P);
}

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
    P.gate_up = (const uint8_t*)layer->d_gate_up;
    P.gate_up_scales = (const uint8_t*)layer->d_gate_up_scales;
    P.down = (const uint8_t*)layer->d_down;
    P.down_scales = (const uint8_t*)layer->d_down_scales;
    P.ld_gate_up = layer->ld_gate_up;
    P.ld_down = layer->ld_down;
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
    P.h = (uint16_t*)(ws + o.h);
    P.z = (float*)(ws + o.z);
    const bool e5m2 = layer->format == ZC_FMT_FP8_E5M2, half = layer->real_type == ZC_REAL_F16;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const cudaError_t e = e5m2 ? (half ? launch_moe<true, true>(P, st) : launch_moe<true, false>(P, st))
                               : (half ? launch_moe<false, true>(P, st) : launch_moe<false, false>(P, st));
    return e == cudaSuccess ? ZC_OK : ZC_E_CUDA;
}

}  // extern "C"
