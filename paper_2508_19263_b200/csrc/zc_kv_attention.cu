// Attention over a quantised key/value cache.
//
// The simplest kernel that is right: a warp has a row and a query head; a lane has a token of 32 for the products with the query, then a
// 32nd of the head's width for the sum of the values.  Running maximum and sum, all in FP32.
#include <type_traits>

#include "zc_kv.cuh"

namespace zc {

struct AttentionParams {
    KvCache C;
    KvBatch B;
    KvTensor q, out;
    float* lse;
    uint32_t q_heads, group;
    float scale;
    uint32_t causal, window;
};

constexpr uint32_t kSimpleWarps = 4;

template <typename T, bool FP4, uint32_t DIM>
__global__ void __launch_bounds__(kSimpleWarps * 32) kv_attention_simple_kernel(const AttentionParams P)
{
    __shared__ float s_q[kSimpleWarps][DIM];
    constexpr uint32_t kRowBytes = FP4 ? DIM / 2 : DIM, kBlocks = DIM / kKvBlock, kOwn = DIM / 32;
    grid_wait();
    grid_launch_dependents();
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint64_t item = (uint64_t)blockIdx.x * kSimpleWarps + warp;
    const int row = (int)(item / P.q_heads);
    const uint32_t head = (uint32_t)(item % P.q_heads), kv = head / P.group;
    if ((uint32_t)row >= P.B.n_rows) return;
    const int found = kv_find(P.B, row);
    uint32_t b = found < 0 ? 0 : (uint32_t)found;
    int pos;
    if (!kv_position(P.B, row, b, pos)) return;
    const int len = kv_len(P.B, b), to = P.causal ? pos + 1 : len, from = P.window ? max(0, to - (int)min(P.window, 0x7FFFFFFFu)) : 0;
    const T* q = reinterpret_cast<const T*>(P.q.d + (uint64_t)row * P.q.ld_row + head * P.q.ld_head);
    for (uint32_t i = lane; i < DIM; i += 32) s_q[warp][i] = (float)q[i];
    __syncwarp();
    float top = -INFINITY, sum = 0.0f, acc[kOwn] = {};
    for (int t0 = from / 32 * 32; t0 < to; t0 += 32) {
        const int t = t0 + (int)lane;
        int page = t >= from && t < to ? kv_page(P.C, P.B, b, (uint32_t)t >> P.C.page_shift) : -1;
        const uint64_t at = page < 0 ? 0 : ((((uint64_t)page * P.C.heads + kv) << P.C.page_shift) + (t & ((1 << P.C.page_shift) - 1)));
        float x = -INFINITY;
        if (page >= 0) {
            const uint32_t* w = reinterpret_cast<const uint32_t*>(P.C.elems[0] + at * kRowBytes);
            x = 0.0f;
            for (uint32_t k = 0; k < kBlocks; ++k) {
                float part = 0.0f;
                for (uint32_t i = 0; i < kRowBytes / kBlocks / 4; ++i) {
                    uint32_t h[4];
                    const uint32_t word = w[k * (kRowBytes / kBlocks / 4) + i];
                    if (FP4) fp4_to_half(word, h);
                    else e4m3_to_half(word, h);
                    for (uint32_t j = 0; j < (FP4 ? 4 : 2); ++j) {
                        const float2 e = half_pair(h[j]);
                        const uint32_t d = k * kKvBlock + i * (FP4 ? 8 : 4) + 2 * j;
                        part = fmaf(e.x, s_q[warp][d], fmaf(e.y, s_q[warp][d + 1], part));
                    }
                }
                x = fmaf(part, e8m0_value(P.C.scales[0][at * kBlocks + k]), x);
            }
            x *= P.scale;
        }
        float best = x;
        for (int d = 16; d; d >>= 1) best = fmaxf(best, __shfl_xor_sync(0xFFFFFFFFu, best, d));
        const bool bad = __any_sync(0xFFFFFFFFu, x != x);
        const float next = fmaxf(top, best);
        if (next == -INFINITY && !bad) continue;
        const float shrink = top == -INFINITY ? 0.0f : expf(top - next), p = page >= 0 ? expf(x - next) : 0.0f;
        top = next;
        sum = sum * shrink + p;
        for (uint32_t i = 0; i < kOwn; ++i) acc[i] *= shrink;
        for (int j = 0; j < 32; ++j) {
            const uint64_t there = __shfl_sync(0xFFFFFFFFu, at, j);
            const float pj = __shfl_sync(0xFFFFFFFFu, p, j);
            if (__shfl_sync(0xFFFFFFFFu, page, j) < 0) continue;
            const uint32_t d = lane * kOwn;                                      // within a block: 2 or 4 of 32
            const float s = e8m0_value(P.C.scales[1][there * kBlocks + d / kKvBlock]);
            const uint32_t byte = FP4 ? d / 2 : d;
            const uint32_t word = *reinterpret_cast<const uint32_t*>(P.C.elems[1] + there * kRowBytes + byte / 4 * 4) >> (8 * (byte & 3));
            uint32_t h[4];
            if (FP4) fp4_to_half(word, h);
            else e4m3_to_half(word, h);
            for (uint32_t i = 0; i < kOwn; i += 2) {
                const float2 v = half_pair(h[i / 2]);
                acc[i] = fmaf(pj, v.x * s, acc[i]);
                acc[i + 1] = fmaf(pj, v.y * s, acc[i + 1]);
            }
        }
    }
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
    T* out = reinterpret_cast<T*>(P.out.d + (uint64_t)row * P.out.ld_row + head * P.out.ld_head);
    for (uint32_t i = 0; i < kOwn; ++i) out[lane * kOwn + i] = T(sum == 0.0f ? 0.0f : acc[i] / sum);
    if (P.lse && lane == 0) P.lse[(uint64_t)row * P.q_heads + head] = sum == 0.0f ? -INFINITY : top + logf(sum);
}

}  // namespace zc

using namespace zc;

extern "C" {

size_t zc_kv_attention_workspace_bytes(const zc_kv_cache* cache, const zc_kv_batch* batch, uint32_t q_heads)
{
    if (check_cache(cache) || check_batch(cache, batch) || q_heads == 0 || q_heads % cache->kv_heads || q_heads / cache->kv_heads > ZC_KV_MAX_GROUP) return 0;
    return 256;
}

zc_status zc_kv_attention(const zc_kv_cache* cache, const zc_kv_batch* batch, const zc_kv_attention_args* args, void* d_workspace,
                          size_t workspace_bytes, void* cuda_stream)
{
    if (!args) return ZC_E_INVALID_ARG;
    if (args->type != ZC_REAL_BF16 && args->type != ZC_REAL_F16) return ZC_E_UNSUPPORTED;
    if (const zc_status s = check_cache(cache)) return s;
    if (const zc_status s = check_batch(cache, batch)) return s;
    if (args->q_heads == 0 || args->q_heads % cache->kv_heads || args->causal > 1 || (args->window && !args->causal) || !(fabsf(args->scale) <= 3.402823466e38f)) return ZC_E_INVALID_ARG;
    if (args->q_heads / cache->kv_heads > ZC_KV_MAX_GROUP) return ZC_E_TOO_LARGE;
    if (batch->n_seqs == 0 || batch->n_rows == 0) return ZC_OK;
    for (const zc_kv_tensor* t : {&args->q, &args->out})
        if (const zc_status s = check_tensor(t, 2, batch->n_rows, args->q_heads, cache->head_dim)) return s;
    if (reinterpret_cast<uintptr_t>(args->d_lse) % 4 || !d_workspace || reinterpret_cast<uintptr_t>(d_workspace) % 256) return ZC_E_INVALID_ARG;
    if (batch->n_rows * args->q_heads >= (1ull << 32)) return ZC_E_TOO_LARGE;
    if (workspace_bytes < zc_kv_attention_workspace_bytes(cache, batch, args->q_heads)) return ZC_E_BUFFER_TOO_SMALL;
    unsigned int* marks = kv_marks_word();
    if (!marks) return ZC_E_CUDA;
    AttentionParams P{};
    P.C = device_cache(cache);
    P.B = device_batch(cache, batch, marks);
    P.q = device_tensor(&args->q, 2);
    P.out = device_tensor(&args->out, 2);
    P.lse = args->d_lse;
    P.q_heads = args->q_heads;
    P.group = args->q_heads / cache->kv_heads;
    P.scale = args->scale;
    P.causal = args->causal;
    P.window = args->window;
    auto run = [&](auto value, auto fp4, auto dim) {
        cudaLaunchConfig_t cfg{};
        cudaLaunchAttribute at[1] = {launch_early()};
        cfg.blockDim = dim3(kSimpleWarps * 32);
        cfg.gridDim = dim3((uint32_t)ceil_div((uint64_t)P.B.n_rows * P.q_heads, kSimpleWarps));
        cfg.stream = (cudaStream_t)cuda_stream;
        cfg.attrs = at;
        cfg.numAttrs = 1;
        return cudaLaunchKernelEx(&cfg, kv_attention_simple_kernel<decltype(value), decltype(fp4)::value, decltype(dim)::value>, P);
    };
    auto dims = [&](auto value, auto fp4) {
        return cache->head_dim == 128 ? run(value, fp4, std::integral_constant<uint32_t, 128>()) : run(value, fp4, std::integral_constant<uint32_t, 64>());
    };
    auto formats = [&](auto value) { return cache->format == ZC_FMT_FP4_E2M1 ? dims(value, std::true_type()) : dims(value, std::false_type()); };
    const cudaError_t e = args->type == ZC_REAL_BF16 ? formats(__nv_bfloat16()) : formats(__half());
    return e == cudaSuccess ? ZC_OK : ZC_E_CUDA;
}

}  // extern "C"
