// zc_fp8_matmul: D = A B^T of FP8 matrices with a scale byte per 128 columns, on the fifth-generation tensor cores.
//
// The instruction that takes FP8 operands with E8M0 scales multiplies 32 columns at a time and looks up one scale byte per
// row of A and of B in tensor memory.  A scale byte that holds for 128 columns is simply looked up by four instructions in
// a row, so the bytes go into the product as they are stored, four of them (512 columns) to a 32-bit word of tensor memory,
// and no accumulator ever leaves tensor memory before the sum over k is complete.
//
// Roles of a thread block's warps: 0 copies tiles of 128 rows x 128 bytes into shared memory (tensor copies, 128-byte
// swizzle; what lies outside of a matrix arrives as zeros), 1 issues the matrix instructions, 4-7 bring the accumulators
// to memory, 8-11 bring the scale bytes into shared memory.
#include "zc_fp8_tensor.cuh"

namespace zc {

constexpr int kMmThreads = 384;
constexpr uint32_t kTile = 128;                  // rows of A, or of B, that a block copies per step
constexpr uint32_t kStepBytes = 128;             // columns per step = bytes of the swizzle = columns of a scale byte
constexpr uint32_t kTileBytes = kTile * kStepBytes;

struct MatmulParams {
    const uint8_t *sa, *sb;                      // scale bytes
    uint64_t ld_sa, ld_sb;
    uint8_t* out;
    uint64_t ld_out;                             // bytes
    uint32_t m, n, steps;                        // rows of A, rows of B, steps of 128 columns
    uint32_t square_a, square_b;                 // 128 rows share a scale byte
    uint32_t idesc;                              // instruction descriptor without the scale selectors
    uint32_t out_type, accumulate, out_wide;     // out_wide: every row of D begins on a 16-byte boundary
    uint32_t tiles_m, tiles_n;
    // Rows of A and of B that a copy of the small kernel brings: no more than there are.  Rows beyond the matrix would arrive as zeros, in
    // the copy engine's time; left out, their accumulators hold whatever comes of what lay in shared memory, and nobody reads them.
    uint32_t rows_a, rows_b;
    uint32_t stages;                             // of the small kernel
    uint32_t by_copy;                            // the large kernel's results leave by tensor copies
    uint32_t spin_limit, skip_copy, skip_math;
};

// The scale words of four steps are a warp's own work, in turn with three others: each has the time of sixteen steps for the
// latency of its loads, a buffer in shared memory, and sees every phase of the buffer's barrier.  (All four warps loading all
// words straight into their quarters of tensor memory, a word ahead: 8192 x 14336 x 4096 took 498 us in short runs, 349 so.)  Tensor
// memory has two sets of words.
constexpr uint32_t kScaleBufs = 4;
constexpr uint32_t kScaleBufBytes = 512 + 1024;  // 128 rows of A, up to 256 of B

// Shared memory behind the operand stages and the scale words.
struct MatmulShared {
    uint64_t full[8], empty[8];
    uint64_t sf_full[kScaleBufs], sf_empty[kScaleBufs];
    uint64_t acc_full[2], acc_empty[1], settled;
    uint32_t tmem, failed, unsettled;            // unsettled: copies or matrix instructions that this block did not see the end of
    uint32_t copied;                             // steps whose copies the block has started
};


template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }

// 16 bytes of consecutive values of D; they exist and are aligned.
template <typename T>
__device__ __forceinline__ void put_wide(uint8_t* row, uint32_t col, const float* v, uint32_t accumulate)
{
    constexpr int PER = 16 / sizeof(T);
    T* p = reinterpret_cast<T*>(row) + col;
    union { uint4 q; T t[PER]; } x;
    if (accumulate) x.q = *reinterpret_cast<const uint4*>(p);
#pragma unroll
    for (int j = 0; j < PER; ++j) x.t[j] = from_float<T>(accumulate ? v[j] + to_float(x.t[j]) : v[j]);
    *reinterpret_cast<uint4*>(p) = x.q;
}
__device__ __forceinline__ void put_wide(const MatmulParams& P, uint32_t row, uint32_t col, const float* v)
{
    uint8_t* r = P.out + (uint64_t)row * P.ld_out;
    if (P.out_type == ZC_REAL_F32) put_wide<float>(r, col, v, P.accumulate);
    else if (P.out_type == ZC_REAL_BF16) put_wide<__nv_bfloat16>(r, col, v, P.accumulate);
    else put_wide<__half>(r, col, v, P.accumulate);
}

// The small kernel's sums from shared memory without an alignment to count on: a column a thread, so that a warp's stores lie next to
// each other, eight at a time.  `width` is a power of two.
template <typename T>
__device__ __forceinline__ void put_columns(const MatmulParams& P, uint32_t base, uint32_t rows, uint32_t width, uint32_t c0, uint32_t m0, uint32_t n0)
{
    const uint32_t shift = 31 - __clz(width);
    for (uint32_t first = threadIdx.x; first < rows * width; first += 8 * kMmThreads) {
        float x[8];
        T* p[8];
#pragma unroll
        for (uint32_t q = 0; q < 8; ++q) {
            const uint32_t i = first + q * kMmThreads, row = i >> shift, col = c0 + (i & (width - 1));
            p[q] = nullptr;
            if (row >= rows || n0 + col >= P.n) continue;
            p[q] = reinterpret_cast<T*>(P.out + (uint64_t)(m0 + row) * P.ld_out) + n0 + col;
            x[q] = __uint_as_float(lds32(base + row * 512 + (((col >> 2) ^ (row & 31)) << 4) + (col & 3) * 4));
        }
#pragma unroll
        for (uint32_t q = 0; q < 8; ++q)
            if (p[q] && P.accumulate) x[q] += to_float(*p[q]);
#pragma unroll
        for (uint32_t q = 0; q < 8; ++q)
            if (p[q]) *p[q] = from_float<T>(x[q]);
    }
}

// One tile of 128 x 128 per block, one after the other along the grid's first axis (the only one with room for all rows that a matrix may
// have); the `gridDim.z` blocks of a cluster share a tile, each takes a part of the steps, and the parts are added up through the
// cluster's shared memory in the order of the ranks.
constexpr size_t small_smem(uint32_t stages) { return 1024 + stages * 2 * kTileBytes + kScaleBufs * kScaleBufBytes + sizeof(MatmulShared); }
constexpr uint32_t kSmallCols = 256;             // tensor memory: 128 accumulator columns, then two sets of 4 + 4 scale columns
constexpr uint32_t kSmallScales = 128;

__global__ void __launch_bounds__(kMmThreads)
matmul_small_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ MatmulParams P)
{
    extern __shared__ uint8_t raw[];
    const uint32_t stages = P.stages;
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t words_at = base + stages * 2 * kTileBytes;
    MatmulShared* S = reinterpret_cast<MatmulShared*>(raw + (words_at - smem_u32(raw)) + kScaleBufs * kScaleBufBytes);
    const uint32_t warp = warp_index(), lane = threadIdx.x & 31;
    const uint32_t parts = gridDim.z, part = blockIdx.z;
    const uint32_t tile_m = blockIdx.x / P.tiles_n, m0 = tile_m * kTile, n0 = (blockIdx.x - tile_m * P.tiles_n) * kTile;
    const uint32_t lo = (uint32_t)((uint64_t)P.steps * part / parts), hi = (uint32_t)((uint64_t)P.steps * (part + 1) / parts);
    const Waiter wait{P.spin_limit, &S->failed};

    if (warp == 0 && lane == 0) {
        prefetch_map(&map_a);
        prefetch_map(&map_b);
        for (uint32_t i = 0; i < stages; ++i) { bar_init(smem_u32(&S->full[i]), 1); bar_init(smem_u32(&S->empty[i]), 1); }
        for (uint32_t i = 0; i < kScaleBufs; ++i) { bar_init(smem_u32(&S->sf_full[i]), 1); bar_init(smem_u32(&S->sf_empty[i]), 1); }
        bar_init(smem_u32(&S->acc_full[0]), 1);
        S->failed = S->unsettled = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc<1>(smem_u32(&S->tmem), kSmallCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = S->tmem;
    grid_wait();                                 // what the kernels before this one wrote is there
    grid_launch_dependents();

    uint32_t st = 0, round = 0;
    if (warp == 0) {
        for (uint32_t i = lo; i < hi; ++i) {
            if (round && !wait.warp(smem_u32(&S->empty[st]), (round - 1) & 1)) break;
            const uint32_t bar = smem_u32(&S->full[st]);
            if (elect_one()) {
                bar_expect(bar, (P.rows_a + P.rows_b) * kStepBytes);
                if (!P.skip_copy) {
                    tensor_copy<1>(base + st * 2 * kTileBytes, &map_a, (int)(i * kStepBytes), (int)m0, bar);
                    tensor_copy<1>(base + st * 2 * kTileBytes + kTileBytes, &map_b, (int)(i * kStepBytes), (int)n0, bar);
                }
            }
            if (++st == stages) { st = 0; ++round; }
        }
    } else if (warp == 1 && !P.skip_math) {
        for (uint32_t i = 0; i < hi - lo; ++i) {
            const uint32_t word = i >> 2, buf = word % kScaleBufs;
            const uint32_t sfa = tmem + kSmallScales + (word & 1) * 8, sfb = sfa + 4;
            const bool fresh = (i & 3) == 0;
            if (!wait.warp(smem_u32(&S->full[st]), round & 1)) break;
            if (fresh) {
                if (!wait.warp(smem_u32(&S->sf_full[buf]), (word / kScaleBufs) & 1)) break;
                // the set's words of eight steps ago are not looked up any more
                if (word >= 2 && !wait.warp(smem_u32(&S->sf_empty[(word - 2) % kScaleBufs]), ((word - 2) / kScaleBufs) & 1)) break;
            }
            tc_fence_after();
            const uint64_t da = operand_desc(base + st * 2 * kTileBytes), db = operand_desc(base + st * 2 * kTileBytes + kTileBytes);
            const uint32_t idesc = P.idesc | ((i & 3) << 29) | ((i & 3) << 4);
            if (elect_one()) {
                if (fresh) {
                    tmem_copy_scales<1>(sfa, words_at + buf * kScaleBufBytes);
                    tmem_copy_scales<1>(sfb, words_at + buf * kScaleBufBytes + 512);
                }
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j) mma_scaled<1>(tmem, da + 2 * j, db + 2 * j, idesc, sfa, sfb, i | j);
                mma_commit<1>(smem_u32(&S->empty[st]));
                if ((i & 3) == 3) mma_commit<1>(smem_u32(&S->sf_empty[buf]));
            }
            __syncwarp();
            if (++st == stages) { st = 0; ++round; }
        }
        if (elect_one()) mma_commit<1>(smem_u32(&S->acc_full[0]));
    } else if (warp >= 8) {
        const uint32_t buf = warp - 8, at = words_at + buf * kScaleBufBytes + lane * 16;
        for (uint32_t i = lo + 4 * buf, k = 0; i < hi; i += 4 * kScaleBufs, ++k) {
            uint32_t a[4], b[4];
#pragma unroll
            for (uint32_t q = 0; q < 4; ++q) {
                a[q] = scale_word(P.sa, P.ld_sa, P.square_a, m0 + 32 * q + lane, P.m, i, hi);
                b[q] = scale_word(P.sb, P.ld_sb, P.square_b, n0 + 32 * q + lane, P.n, i, hi);
            }
            if (!__all_sync(0xFFFFFFFFu, k == 0 || wait(smem_u32(&S->sf_empty[buf]), (k - 1) & 1))) break;
            sts128(at, a);
            sts128(at + 512, b);
            fence_async_shared();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_u32(&S->sf_full[buf]));
        }
    }
    __syncwarp();
    const uint32_t rows = P.m - m0 < kTile ? P.m - m0 : kTile;
    if (warp >= 4 && warp < 8) {
        const uint32_t quad = warp & 3, row = quad * 32 + lane;
        if (__all_sync(0xFFFFFFFFu, wait(smem_u32(&S->acc_full[0]), 0) && !*wait.failed) && quad * 32 < rows) {
            tc_fence_after();
            for (uint32_t c = 0; c < 4; ++c) {
                uint32_t v[32];
                tmem_ld32(tmem + (quad * 32u << 16) + c * 32, v);
                // the operand stages are free once the last instruction is done; 16-byte pieces turned by the row
                if (row < rows) {
#pragma unroll
                    for (uint32_t q = 0; q < 8; ++q) sts128(base + row * 512 + (((c * 8 + q) ^ (row & 31)) << 4), v + 4 * q);
                }
            }
            tc_fence_before();
        }
    }
    __syncthreads();
    // Rank r adds up columns 128 r / parts .. of all rows, in the order of the ranks, in its own shared memory, where no other rank
    // reads these columns.
    const uint32_t width = 128 / parts, c0 = part * width, cols = P.n - n0;
    if (parts > 1) {
        cluster_sync();
        const uint32_t pieces = width / 4;
        for (uint32_t i = threadIdx.x; i < rows * pieces; i += kMmThreads) {
            const uint32_t row = i / pieces, piece = c0 / 4 + i - row * pieces;
            const uint32_t at = base + row * 512 + ((piece ^ (row & 31)) << 4);
            float4 x[8];
#pragma unroll
            for (uint32_t r = 0; r < 8; ++r)
                if (r < parts) x[r] = ld_cluster_f4(map_shared(at, r));
#pragma unroll
            for (uint32_t r = 1; r < 8; ++r)
                if (r < parts) { x[0].x += x[r].x; x[0].y += x[r].y; x[0].z += x[r].z; x[0].w += x[r].w; }
            const uint32_t s[4] = {__float_as_uint(x[0].x), __float_as_uint(x[0].y), __float_as_uint(x[0].z), __float_as_uint(x[0].w)};
            sts128(at, s);
        }
        __syncthreads();
        cluster_arrive();                        // this block has read all that it needs of the others
    }
    const uint32_t per = P.out_type == ZC_REAL_F32 ? 4 : 8;
    if (P.out_wide && (cols >= 128 || cols % per == 0)) {
        const uint32_t units = width / per;
        for (uint32_t i = threadIdx.x; i < rows * units; i += kMmThreads) {
            const uint32_t row = i / units, col = c0 + (i - row * units) * per, piece = col >> 2;
            if (col >= cols) continue;
            uint4 v[2];
            v[0] = lds128(base + row * 512 + ((piece ^ (row & 31)) << 4));
            if (per == 8) v[1] = lds128(base + row * 512 + (((piece + 1) ^ (row & 31)) << 4));
            put_wide(P, m0 + row, n0 + col, reinterpret_cast<const float*>(v));
        }
    } else {
        if (P.out_type == ZC_REAL_F32) put_columns<float>(P, base, rows, width, c0, m0, n0);
        else if (P.out_type == ZC_REAL_BF16) put_columns<__nv_bfloat16>(P, base, rows, width, c0, m0, n0);
        else put_columns<__half>(P, base, rows, width, c0, m0, n0);
    }
    if (*wait.failed) {                          // whichever role gave up: see what copies and instructions are still under way
        if (warp == 0 && !P.skip_copy && !settled_stage(smem_u32(S->full), lane, stages, st, round, P.spin_limit)) S->unsettled = 1;
        if (warp == 1 && lane == 0 && !P.skip_math && !settled(smem_u32(&S->acc_full[0]), 0, P.spin_limit)) S->unsettled = 1;
        __syncthreads();
        if (threadIdx.x == 0) report(S->unsettled);
    }
    __syncthreads();
    if (parts > 1) cluster_wait();               // no other block reads from this one any more
    if (warp == 1) tmem_free<1>(tmem, kSmallCols);
}

// Tiles of 256 x 256 per pair of blocks: each block holds 128 rows of A and 128 of B, the matrix instruction of the pair reads
// both blocks' shared memory, and each block ends with 128 x 256 accumulators.  Two accumulators of 256 columns and the scale
// words do not fit into 512 columns of tensor memory side by side, so the two overlap by 32 columns: the result warps empty these
// first, and the next tile's instructions begin when they have, while the other 224 columns are still on their way out.
constexpr uint32_t kLargeStages = 6;
constexpr uint32_t kResultBytes = 32 * 64;       // what a warp sends off at a time: 32 rows x 64 bytes
constexpr uint32_t kResultBufs = 3;              // per warp
constexpr size_t kLargeSmem = 1024 + kLargeStages * 2 * kTileBytes + 4 * kResultBufs * kResultBytes + kScaleBufs * kScaleBufBytes + sizeof(MatmulShared);
constexpr uint32_t kLargeCols = 512, kLargeSecond = 224, kLargeScales = 480;     // two sets of 4 + 8 scale columns
constexpr uint32_t kSwath = 8;                   // rows of tiles that are walked through together, column by column

template <typename T>
__device__ __forceinline__ uint32_t pack_pair(const uint32_t v[2])
{
    union { T t[2]; uint32_t w; } x;
    x.t[0] = from_float<T>(__uint_as_float(v[0]));
    x.t[1] = from_float<T>(__uint_as_float(v[1]));
    return x.w;
}
// A warp's 32 rows of 64 bytes, a row per lane, into the next of its buffers and off; what was sent from there last has been read
// by then.
__device__ __forceinline__ void send(const CUtensorMap& map, uint32_t buffer, uint32_t lane, int x, int y, const uint32_t w[16])
{
    const bool one = elect_one();                // the same lane every time: groups are a thread's own
    if (one) tensor_store_wait_read<kResultBufs - 1>();
    __syncwarp();
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) sts128(buffer + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4), w + 4 * j);
    fence_async_shared();
    __syncwarp();
    if (one) tensor_store(&map, x, y, buffer);
}

// The same without an alignment to count on, or with D to be added to: 16 columns in FP32 at a time through shared memory, so that half a
// warp's stores lie next to each other, and sixteen reads, then sixteen stores, on their way at once.
template <typename T>
__device__ __forceinline__ void put_rows(const MatmulParams& P, uint32_t buffer, uint32_t lane, uint32_t row0, uint32_t col0, const uint32_t v[32])
{
    const uint32_t e = lane & 15, odd = lane >> 4;
#pragma unroll
    for (uint32_t half = 0; half < 2; ++half) {
        const uint32_t col = col0 + half * 16 + e, n = col < P.n ? min(P.m - row0, 32u) : 0;
        __syncwarp();
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) sts128(buffer + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4), v + half * 16 + 4 * j);
        __syncwarp();
        float x[16];
#pragma unroll
        for (uint32_t i = 0; i < 16; ++i) x[i] = __uint_as_float(lds32(buffer + (2 * i + odd) * 64 + (((e >> 2) ^ (i & 3)) << 4) + (e & 3) * 4));
        uint8_t* p = P.out + (uint64_t)(row0 + odd) * P.ld_out;
        if (P.accumulate) {
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i)
                if (2 * i + odd < n) x[i] += to_float(reinterpret_cast<const T*>(p + 2 * i * P.ld_out)[col]);
        }
#pragma unroll
        for (uint32_t i = 0; i < 16; ++i)
            if (2 * i + odd < n) reinterpret_cast<T*>(p + 2 * i * P.ld_out)[col] = from_float<T>(x[i]);
    }
}

__device__ __forceinline__ void large_tile(const MatmulParams& P, uint32_t i, uint32_t& m, uint32_t& n)
{
    const uint32_t per = kSwath * P.tiles_n, swath = i / per, first = swath * kSwath;
    const uint32_t height = min(P.tiles_m - first, kSwath), in = i - swath * per;
    n = in / height;
    m = first + in - n * height;
}

__global__ void __launch_bounds__(kMmThreads, 1)
matmul_large_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_d,
                    const __grid_constant__ MatmulParams P)
{
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t results_at = base + kLargeStages * 2 * kTileBytes, words_at = results_at + 4 * kResultBufs * kResultBytes;
    MatmulShared* S = reinterpret_cast<MatmulShared*>(raw + (words_at - smem_u32(raw)) + kScaleBufs * kScaleBufBytes);
    const uint32_t warp = warp_index(), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank(), pair = blockIdx.x >> 1, pairs = gridDim.x >> 1, tiles = P.tiles_m * P.tiles_n;
    const Waiter wait{P.spin_limit, &S->failed, map_shared(smem_u32(&S->failed), rank ^ 1)};

    if (warp == 0 && lane == 0) {
        prefetch_map(&map_a);
        prefetch_map(&map_b);
        for (uint32_t i = 0; i < kLargeStages; ++i) { bar_init(smem_u32(&S->full[i]), 1); bar_init(smem_u32(&S->empty[i]), 1); }
        for (uint32_t i = 0; i < kScaleBufs; ++i) { bar_init(smem_u32(&S->sf_full[i]), 2); bar_init(smem_u32(&S->sf_empty[i]), 1); }
        for (uint32_t i = 0; i < 2; ++i) bar_init(smem_u32(&S->acc_full[i]), 1);
        bar_init(smem_u32(&S->acc_empty[0]), 8);
        bar_init(smem_u32(&S->settled), 1);
        S->failed = S->unsettled = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc<2>(smem_u32(&S->tmem), kLargeCols);
    tc_fence_before();
    __syncthreads();
    cluster_sync();                              // the pair's barriers are there before either block uses them
    tc_fence_after();
    const uint32_t tmem = S->tmem;
    grid_wait();                                 // what the kernels before this one wrote is there
    grid_launch_dependents();

    if (warp == 0) {
        // both blocks copy their halves; the bytes count on the first block's barrier
        uint32_t st = 0, round = 0;
        bool ok = true;
        for (uint32_t i = pair; i < tiles && ok; i += pairs) {
            uint32_t tm, tn;
            large_tile(P, i, tm, tn);
            const int row_a = (int)(tm * 256 + rank * 128), row_b = (int)(tn * 256 + rank * 128);
            for (uint32_t k = 0; k < P.steps; ++k) {
                if (!(ok = round == 0 || wait.warp(smem_u32(&S->empty[st]), (round - 1) & 1))) break;
                const uint32_t bar = map_shared(smem_u32(&S->full[st]), 0), to = base + st * 2 * kTileBytes;
                if (elect_one()) {
                    if (rank == 0) bar_expect(smem_u32(&S->full[st]), 4 * kTileBytes);
                    if (!P.skip_copy) {
                        tensor_copy<2>(to, &map_a, (int)(k * kStepBytes), row_a, bar);
                        tensor_copy<2>(to + kTileBytes, &map_b, (int)(k * kStepBytes), row_b, bar);
                    }
                }
                if (++st == kLargeStages) { st = 0; ++round; }
            }
        }
        if (lane == 0) S->copied = round * kLargeStages + st;
    } else if (warp == 1 && rank == 0 && !P.skip_math) {
        uint32_t st = 0, round = 0, word = 0, tile = 0;
        bool ok = true;
        for (uint32_t i = pair; i < tiles && ok; i += pairs, ++tile) {
            const uint32_t d = tmem + (tile & 1 ? kLargeSecond : 0);
            // the columns that this tile's accumulator shares with the one before it are empty, and with them all of the one before that
            if (tile && !(ok = wait.warp_across(smem_u32(&S->acc_empty[0]), (tile - 1) & 1))) break;
            for (uint32_t k = 0; k < P.steps; ++k) {
                const uint32_t buf = word % kScaleBufs, sfa = tmem + kLargeScales + (word & 1) * 12, sfb = sfa + 4;
                const bool fresh = (k & 3) == 0, last = (k & 3) == 3 || k + 1 == P.steps;
                if (!(ok = wait.warp(smem_u32(&S->full[st]), round & 1))) break;
                if (fresh) {
                    if (!(ok = wait.warp_across(smem_u32(&S->sf_full[buf]), (word / kScaleBufs) & 1))) break;
                    // the set's words of two before are not looked up any more
                    if (word >= 2 && !(ok = wait.warp(smem_u32(&S->sf_empty[(word - 2) % kScaleBufs]), ((word - 2) / kScaleBufs) & 1))) break;
                }
                tc_fence_after();
                const uint64_t da = operand_desc(base + st * 2 * kTileBytes), db = operand_desc(base + st * 2 * kTileBytes + kTileBytes);
                const uint32_t idesc = P.idesc | ((k & 3) << 29) | ((k & 3) << 4), from = words_at + buf * kScaleBufBytes;
                if (elect_one()) {
                    if (fresh) {
                        tmem_copy_scales<2>(sfa, from);
                        tmem_copy_scales<2>(sfb, from + 512);
                        tmem_copy_scales<2>(sfb + 4, from + 1024);
                    }
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j) mma_scaled<2>(d, da + 2 * j, db + 2 * j, idesc, sfa, sfb, k | j);
                    mma_commit<2>(smem_u32(&S->empty[st]));
                    if (last) mma_commit<2>(smem_u32(&S->sf_empty[buf]));
                }
                __syncwarp();
                word += last;
                if (++st == kLargeStages) { st = 0; ++round; }
            }
            if (elect_one()) mma_commit<2>(smem_u32(&S->acc_full[tile & 1]));
            __syncwarp();
        }
    } else if (warp >= 8) {
        // this block's 128 rows of A and the pair's 256 of B
        const uint32_t buf = warp - 8, at = words_at + buf * kScaleBufBytes + lane * 16, per = (P.steps + 3) >> 2;
        uint32_t round = 0;
        for (uint32_t w = buf, i = pair; i < tiles; w += kScaleBufs, ++round) {
            while (w >= per && i < tiles) { w -= per; i += pairs; }
            if (i >= tiles) break;
            uint32_t tm, tn, a[4], b[8];
            large_tile(P, i, tm, tn);
#pragma unroll
            for (uint32_t q = 0; q < 4; ++q) a[q] = scale_word(P.sa, P.ld_sa, P.square_a, tm * 256 + rank * 128 + 32 * q + lane, P.m, 4 * w, P.steps);
#pragma unroll
            for (uint32_t q = 0; q < 8; ++q) b[q] = scale_word(P.sb, P.ld_sb, P.square_b, tn * 256 + 32 * q + lane, P.n, 4 * w, P.steps);
            if (!__all_sync(0xFFFFFFFFu, round == 0 || wait(smem_u32(&S->sf_empty[buf]), (round - 1) & 1))) break;
            sts128(at, a);
            sts128(at + 512, b);
            sts128(at + 1024, b + 4);
            fence_async_shared();
            __syncwarp();
            if (lane == 0) bar_arrive_cluster(map_shared(smem_u32(&S->sf_full[buf]), 0));
        }
    } else if (warp >= 4) {
        const uint32_t quad = warp & 3;
        uint32_t tile = 0, sent = 0;
        for (uint32_t i = pair; i < tiles; i += pairs, ++tile) {
            uint32_t tm, tn;
            large_tile(P, i, tm, tn);
            if (!__all_sync(0xFFFFFFFFu, wait(smem_u32(&S->acc_full[tile & 1]), (tile >> 1) & 1) && !*wait.failed)) break;
            tc_fence_after();
            const uint32_t d = tmem + (quad * 32u << 16) + (tile & 1 ? kLargeSecond : 0), results = results_at + quad * kResultBufs * kResultBytes;
#pragma unroll 1
            for (uint32_t q = 0; q < 8; ++q) {
                const uint32_t c = tile & 1 ? q : (q + 7) & 7;           // the shared columns first
                uint32_t v[32];
                tmem_ld32(d + c * 32, v);
                if (q == 0) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive_cluster(map_shared(smem_u32(&S->acc_empty[0]), 0));
                }
                if (P.by_copy) {
                    // rows of 64 bytes through shared memory: stores of 16 bytes to 32 rows at a time cost a tenth of the whole product
                    const uint32_t row0 = tm * 256 + rank * 128 + quad * 32, col0 = tn * 256 + c * 32;
                    if (row0 >= P.m || col0 >= P.n) continue;
                    if (P.out_type == ZC_REAL_F32) {
                        send(map_d, results + (sent++ % kResultBufs) * kResultBytes, lane, (int)col0, (int)row0, v);
                        if (col0 + 16 < P.n) send(map_d, results + (sent++ % kResultBufs) * kResultBytes, lane, (int)col0 + 16, (int)row0, v + 16);
                    } else {
                        uint32_t w[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) w[j] = P.out_type == ZC_REAL_BF16 ? pack_pair<__nv_bfloat16>(v + 2 * j) : pack_pair<__half>(v + 2 * j);
                        send(map_d, results + (sent++ % kResultBufs) * kResultBytes, lane, (int)col0, (int)row0, w);
                    }
                } else {
                    const uint32_t row0 = tm * 256 + rank * 128 + quad * 32, col0 = tn * 256 + c * 32;
                    if (row0 >= P.m || col0 >= P.n) continue;
                    if (P.out_type == ZC_REAL_F32) put_rows<float>(P, results, lane, row0, col0, v);
                    else if (P.out_type == ZC_REAL_BF16) put_rows<__nv_bfloat16>(P, results, lane, row0, col0, v);
                    else put_rows<__half>(P, results, lane, row0, col0, v);
                }
            }
        }
        __syncwarp();
        if (elect_one()) tensor_store_wait_read<0>();
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    cluster_sync();                              // nothing of either block arrives at, or is copied into, the other any more
    tc_fence_after();
    if (*wait.failed) {                          // both blocks know of it: but for what they left under way
        if (rank == 0 && warp == 0 && lane == 0 && !P.skip_copy) {
            // the bytes of both count here; where one of them is a few steps ahead, only its own come
            const uint32_t mine = S->copied, other = ld_cluster_u32(map_shared(smem_u32(&S->copied), 1)), n = max(mine, other);
            for (uint32_t i = n > kLargeStages ? n - kLargeStages : 0; i < n; ++i) {
                const uint32_t bar = smem_u32(&S->full[i % kLargeStages]);
                if (i >= mine) bar_expect(bar, 2 * kTileBytes);
                else if (i >= other) bar_forgo(bar, 2 * kTileBytes);
                if (!settled(bar, (i / kLargeStages) & 1, P.spin_limit)) S->unsettled = 1;
            }
        }
        __syncwarp();
        if (warp == 1) {
            if (rank == 0 && elect_one()) mma_commit<2>(smem_u32(&S->settled));
            if (lane == 0 && !settled(smem_u32(&S->settled), 0, P.spin_limit)) S->unsettled = 1;
        }
        __syncwarp();
        __syncthreads();
        if (threadIdx.x == 0) report(S->unsettled);
        __syncwarp();
        cluster_sync();
    }
    if (warp == 1) tmem_free<2>(tmem, kLargeCols);
}

// D = 0 (K = 0): nothing to copy or multiply.
__global__ void zero_kernel(const __grid_constant__ MatmulParams P, uint32_t width)
{
    for (uint64_t r = blockIdx.x; r < P.m; r += gridDim.x)
        for (uint64_t i = threadIdx.x; i < (uint64_t)P.n * width; i += blockDim.x) P.out[r * P.ld_out + i] = 0;
}

// The marks of both files' kernels, read and cleared at once: whatever another stream's kernel leaves is found by this query or by a later
// one.  Every query has a place of its own for its answer, as long as no more than kAnswers threads ask at the same time.
constexpr uint32_t kAnswers = 1024;
static __device__ unsigned int g_answers[kAnswers];
__global__ void collect_kernel(unsigned int* product, unsigned int* layer, uint32_t at) { g_answers[at] = atomicExch(product, 0u) | atomicExch(layer, 0u); }

// From this many tiles of 256 x 256 on, half of the 74 pairs of blocks that the GPU has room for, a product goes to pairs; below, four
// times as many tiles of 128 x 128 fill it better.  Pairs and small tiles, us: 512 x 4096 x 4096 (32 tiles) 16.4 and 14.1, 1024 x 2560 x 4096
// (40) 17.6 and 18.4, 640 x 4096 x 4096 (48) 17.4 and 19.0, 300 x 14336 x 4096 (112) 33.0 and 34.8.  With few steps the start and end of
// the larger tiles count for more, which the rule does not look at: 2048 x 1280 x 2048 (40 tiles, 16 steps) 12.4 and 11.7,
// 1024 x 4096 x 1024 (64 tiles, 8 steps) 9.7 and 8.3.
constexpr uint64_t kPairsFrom = 37;
// A plain launch, which says how it went itself: the runtime's last error may be that of another call.
template <typename... Params, typename... Args>
static cudaError_t launch(void (*kernel)(Params...), uint32_t grid, uint32_t block, cudaStream_t st, Args... args)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.stream = st;
    return cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
}

// Blocks of the large kernel that are on the GPU at once, in whole pairs.
static uint32_t large_blocks()
{
    if (cudaFuncSetAttribute(matmul_large_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kLargeSmem) != cudaSuccess) return 0;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((uint32_t)sm_count() / 2 * 2);
    cfg.blockDim = dim3(kMmThreads);
    cfg.dynamicSmemBytes = kLargeSmem;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {2, 1, 1};
    cfg.attrs = at;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, (const void*)matmul_large_kernel, &cfg) != cudaSuccess || n <= 0) return 0;
    return std::min((uint32_t)n * 2, cfg.gridDim.x);
}

}  // namespace zc

using namespace zc;

extern "C" {

zc_status zc_fp8_matmul(const zc_fp8_matrix* a, const zc_fp8_matrix* b, zc_real out_type, void* d_out, uint64_t ld_out,
                        uint32_t accumulate, void* cuda_stream)
{
    if (const zc_status s = check_matrix(a)) return s;
    if (const zc_status s = check_matrix(b)) return s;
    const uint32_t width = real_bytes(out_type);
    if (!width) return ZC_E_UNSUPPORTED;
    if (a->cols != b->cols) return ZC_E_INVALID_ARG;
    if (a->rows == 0 || b->rows == 0) return ZC_OK;
    if (!d_out || reinterpret_cast<uintptr_t>(d_out) % width || ld_out < b->rows || ld_out >= (1ull << 39)) return ZC_E_INVALID_ARG;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    MatmulParams P{};
    P.out = (uint8_t*)d_out;
    P.ld_out = ld_out * width;
    P.m = (uint32_t)a->rows;
    P.n = (uint32_t)b->rows;
    if (a->cols == 0) {
        return accumulate || launch(zero_kernel, (uint32_t)std::min<uint64_t>(P.m, 1024), 256, st, P, width) == cudaSuccess ? ZC_OK : ZC_E_CUDA;
    }
    P.sa = (const uint8_t*)a->d_scales;
    P.sb = (const uint8_t*)b->d_scales;
    P.ld_sa = a->ld_scales;
    P.ld_sb = b->ld_scales;
    P.steps = (uint32_t)ceil_div(a->cols, kStepBytes);
    P.square_a = a->block_rows == 128;
    P.square_b = b->block_rows == 128;
    P.out_type = out_type;
    P.accumulate = accumulate != 0;
    P.out_wide = reinterpret_cast<uintptr_t>(d_out) % 16 == 0 && P.ld_out % 16 == 0;
    P.spin_limit = test_knobs().spin_limit;
    P.skip_copy = test_knobs().skip_copy;
    P.skip_math = test_knobs().skip_math;
    P.tiles_m = (uint32_t)ceil_div(P.m, kTile);
    P.tiles_n = (uint32_t)ceil_div(P.n, kTile);
    const uint64_t tiles = (uint64_t)P.tiles_m * P.tiles_n;
    const uint64_t large = ceil_div(P.m, 256) * ceil_div(P.n, 256);
    // for up to 128 tokens half of a pair's tile would be empty (16 x 14336 x 4096: 21.6 us in pairs, 14.0 in small tiles; 128: 19.2 and 15.4)
    const bool pairs = P.m > 128 && P.n > 128 && large >= kPairsFrom;
    P.rows_a = pairs || P.m >= kTile ? kTile : (uint32_t)round_up(P.m, 8);
    P.rows_b = pairs || P.n >= kTile ? kTile : (uint32_t)round_up(P.n, 8);
    CUtensorMap map_a, map_b;
    if (!make_map(&map_a, a->d_elems, a->rows, a->cols, a->ld_elems, P.rows_a) || !make_map(&map_b, b->d_elems, b->rows, b->cols, b->ld_elems, P.rows_b)) return ZC_E_CUDA;
    if (pairs) {
        static OncePerDevice once;
        const uint32_t blocks = once([] { return large_blocks(); });
        if (!blocks) return ZC_E_CUDA;
        P.tiles_m = (uint32_t)ceil_div(P.m, 256);
        P.tiles_n = (uint32_t)ceil_div(P.n, 256);
        if (large >= (1ull << 31)) return ZC_E_TOO_LARGE;
        P.idesc = instruction_of(a->format, b->format, 256, 256);
        // a copy that runs over the last column is cut off at the next 16 bytes, not at the column: what lies behind it in the
        // row would be overwritten
        P.by_copy = P.out_wide && !P.accumulate && (uint64_t)P.n * width % 16 == 0 && P.ld_out < (1ull << 40);
        CUtensorMap map_d = map_a;
        if (P.by_copy && !make_result_map(&map_d, d_out, out_type, P.m, P.n, P.ld_out)) return ZC_E_CUDA;
        const uint32_t grid = (uint32_t)std::min<uint64_t>(blocks, 2 * large);
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(grid);
        cfg.blockDim = dim3(kMmThreads);
        cfg.dynamicSmemBytes = kLargeSmem;
        cfg.stream = st;
        cudaLaunchAttribute at[2];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim = {2, 1, 1};
        at[1] = launch_early();
        cfg.attrs = at;
        cfg.numAttrs = 2;
        return cudaLaunchKernelEx(&cfg, matmul_large_kernel, map_a, map_b, map_d, P) == cudaSuccess ? ZC_OK : ZC_E_CUDA;
    }
    P.idesc = instruction_of(a->format, b->format, 128, 128);
    // Parts of k as long as there is an SM for each: 1 x 4096 x 4096 takes 12.2 us in 32 blocks, 6.6 in 128; 128 x 4096 x 4096 13.4 and
    // 8.9.  Adding the parts up costs more the more rows there are, so these have 8 steps each at least, few rows 4
    // (1024 x 1024 x 1024, 8 steps: 6.1 us in one part, 7.7 in two).
    uint32_t parts = 1;
    while (parts < 8 && tiles * parts * 2 <= (uint64_t)sm_count() && P.steps >= (P.m > 32 ? 16 : 8) * parts) parts *= 2;
    // one block per SM has all of the shared memory, two have half of it each (64 x 14336 x 4096: 14.4 us, 18.0 with half)
    P.stages = tiles * parts <= (uint64_t)sm_count() ? 6 : 3;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((uint32_t)tiles, 1, parts);    // 2^24 at most: one of the two sides has a tile, or there are few
    cfg.blockDim = dim3(kMmThreads);
    cfg.dynamicSmemBytes = small_smem(P.stages);
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {1, 1, parts};
    at[1] = launch_early();
    cfg.attrs = at;
    cfg.numAttrs = 2;
    static OncePerDevice once;
    if (!once([] { return (uint32_t)(cudaFuncSetAttribute(matmul_small_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)small_smem(6)) == cudaSuccess); })) return ZC_E_CUDA;
    if (cudaLaunchKernelEx(&cfg, matmul_small_kernel, map_a, map_b, P) != cudaSuccess) return ZC_E_CUDA;
    return ZC_OK;
}

zc_status zc_fp8_status(void* cuda_stream)
{
    static std::atomic<uint32_t> asked{0};
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(st, &capture) != cudaSuccess || capture != cudaStreamCaptureStatusNone) return ZC_E_CUDA;
    unsigned int *product = marks_word(), *layer = moe_marks_word(), marks = 0;
    if (!product || !layer) return ZC_E_CUDA;
    const uint32_t at = asked.fetch_add(1, std::memory_order_relaxed) % kAnswers;
    if (launch(collect_kernel, 1, 1, st, product, layer, at) != cudaSuccess) return ZC_E_CUDA;
    if (cudaMemcpyFromSymbolAsync(&marks, g_answers, sizeof marks, at * sizeof marks, cudaMemcpyDeviceToHost, st) != cudaSuccess) return ZC_E_CUDA;
    if (cudaStreamSynchronize(st) != cudaSuccess) return ZC_E_CUDA;
    test_knobs().fp8_marks = marks;
    return marks ? ZC_E_DEVICE_TIMEOUT : ZC_OK;
}

}  // extern "C"
