// Attention over a quantised key/value cache: arguments, choice of kernels, launches.
#include <type_traits>

#include "zc_kv_prompt.cuh"

namespace zc {

// The elements of a cache, a token's head a row, as boxes of up to 32 tokens of a page in the swizzle as wide as a row.
static bool make_cache_map(CUtensorMap* map, const void* elems, uint64_t rows, uint32_t row_bytes, uint32_t box_rows)
{
    const cuuint64_t dims[2] = {row_bytes, rows}, pitch[1] = {row_bytes};
    const cuuint32_t box[2] = {row_bytes, box_rows}, step[2] = {1, 1};
    const CUtensorMapSwizzle swizzle = row_bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : row_bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B;
    return encode_fn() && encode_fn()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(elems), dims, pitch, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                                      CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static uint32_t multiprocessors()
{
    static OncePerDevice once;
    return once([]() -> uint32_t {
        int dev = 0, n = 0;
        return cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess ? (uint32_t)n : 0;
    });
}

// without a device (argument checks): as many as any has
static uint32_t multiprocessors_or_most()
{
    const uint32_t n = multiprocessors();
    return n ? n : 256;
}

// What blocks leave to the joining kernel, and what warps of a block leave to the block.
template <typename S>
static size_t workspace_of(uint32_t blocks, uint32_t early_floats)
{
    return (blocks * sizeof(BlockEnd) + 255) / 256 * 256 + ((size_t)blocks * 2 * S::kCols * (S::kDim + 2) + early_floats) * 4;
}
template <typename S>
static size_t stream_workspace(uint32_t blocks) { return workspace_of<S>(blocks, blocks * S::kWarps * S::kPart); }

template <typename S>
static cudaError_t launch_join(const AttentionParams& P, uint32_t blocks, uint32_t least, cudaLaunchConfig_t cfg)
{
    cfg.gridDim = dim3(blocks, S::kCols < 64 ? S::kCols / 8 : 8u);          // all of them are on the GPU at once
    cfg.blockDim = dim3(256);
    cfg.dynamicSmemBytes = 0;
    return cudaLaunchKernelEx(&cfg, kv_join_kernel<S>, P, blocks, least);
}

template <typename S>
static cudaError_t launch_stream(const AttentionParams& P, const CUtensorMap& keys, const CUtensorMap& values, uint32_t blocks, cudaStream_t st)
{
    static OncePerDevice ready;
    if (!ready([]() -> uint32_t { return cudaFuncSetAttribute(kv_stream_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem) == cudaSuccess; })) return cudaErrorUnknown;
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute at[1] = {launch_early()};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(S::kWarps * 32);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (const cudaError_t e = cudaLaunchKernelEx(&cfg, kv_stream_kernel<S>, P, keys, values)) return e;
    return launch_join<S>(P, blocks, S::kWarps, cfg);
}

template <typename S>
static cudaError_t launch_prompt(const AttentionParams& P, uint32_t blocks, cudaStream_t st)
{
    static OncePerDevice ready;
    if (!ready([]() -> uint32_t {
            return cudaFuncSetAttribute(kv_prompt_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem) == cudaSuccess; })) return cudaErrorUnknown;
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute at[1] = {launch_early()};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(S::kThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (const cudaError_t e = cudaLaunchKernelEx(&cfg, kv_prompt_kernel<S>, P)) return e;
    return launch_join<S>(P, blocks, 1, cfg);
}

// Columns (rows times heads that share a head of the cache) up to which a sequence goes to the kernel of few rows.  That reads and converts the cache once for each 16 of
// them, the other works on 256 whatever there are.  Us of few rows and of many, 8 heads, by columns:
//                                     16 sequences of 6000 tokens       64 of 2000                         one of 32768
//   heads of 128, E4M3   32 and 40:   135, 154 and 179, 157             179, 252 and 248, 254              57, 62 and 76, 62
//                 FP4    48 and 56:   139, 146 and 173, 148             196, 241 and 236, 244              59, 57 and 66, 58
//   heads of 64,  E4M3   64 and 80:   126, 127 and 152, 129             174, 211 and 210, 214              51, 48 and 61, 52
//                 FP4    64 and 80:   122, 120 and 147, 121             166, 204 and 200, 205              50, 47 and 60, 51
static uint32_t few_columns(const zc_kv_cache* c) { return c->head_dim == 64 ? 64 : c->format == ZC_FMT_FP4_E2M1 ? 48 : 32; }

}  // namespace zc

using namespace zc;

extern "C" {

size_t zc_kv_attention_workspace_bytes(const zc_kv_cache* cache, const zc_kv_batch* batch, uint32_t q_heads)
{
    if (check_cache(cache) || check_batch(cache, batch) || q_heads == 0 || q_heads % cache->kv_heads || q_heads / cache->kv_heads > ZC_KV_MAX_GROUP) return 0;
    const uint32_t n = multiprocessors_or_most();
    const bool wide = cache->head_dim == 128;
    size_t bytes = wide ? std::max(stream_workspace<StreamShape<true, 128, 1>>(n), stream_workspace<StreamShape<true, 128, 2>>(n))
                        : std::max(stream_workspace<StreamShape<true, 64, 1>>(n), stream_workspace<StreamShape<true, 64, 2>>(n));
    if ((uint64_t)(q_heads / cache->kv_heads) * std::max(1u, batch->max_new) > few_columns(cache))
        bytes = std::max(bytes, wide ? workspace_of<PromptShape<true, 128>>(n, 0) : workspace_of<PromptShape<true, 64>>(n, 0));
    return bytes;
}

zc_status zc_kv_attention(const zc_kv_cache* cache, const zc_kv_batch* batch, const zc_kv_attention_args* args, void* d_workspace,
                          size_t workspace_bytes, void* cuda_stream)
{
    if (!args) return ZC_E_INVALID_ARG;
    if (args->type != ZC_REAL_BF16 && args->type != ZC_REAL_F16) return ZC_E_UNSUPPORTED;
    if (const zc_status s = check_cache(cache)) return s;
    if (const zc_status s = check_batch(cache, batch)) return s;
    if (args->q_heads == 0 || args->q_heads % cache->kv_heads || args->causal > 1 || (args->window && !args->causal) || !(fabsf(args->scale) <= 2e38f)) return ZC_E_INVALID_ARG;
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
    P.scale_mantissa = 2.0f * (float)frexp((double)args->scale * 1.4426950408889634, &P.scale_exponent);
    if (args->scale == 0.0f) { P.scale_mantissa = 1.0f; P.scale_exponent = -1000; }          // the least that logit_factor gives
    else if (fabsf(P.scale_mantissa) == 2.0f) P.scale_mantissa *= 0.5f;
    else --P.scale_exponent;
    P.causal = args->causal;
    P.window = args->window;
    P.workspace = (uint8_t*)d_workspace;
    P.half_type = args->type == ZC_REAL_F16;
    P.q_wide = reinterpret_cast<uintptr_t>(P.q.d) % 8 == 0 && P.q.ld_row % 8 == 0 && P.q.ld_head % 8 == 0;
    P.out_wide = reinterpret_cast<uintptr_t>(P.out.d) % 8 == 0 && P.out.ld_row % 8 == 0 && P.out.ld_head % 8 == 0;
    P.most_rows = 0xFFFFFFFFu;
    P.spin_limit = test_knobs().spin_limit;
    P.skip_copy = test_knobs().skip_copy;
    P.skip_math = test_knobs().skip_math;
    const uint32_t blocks = multiprocessors();
    if (!blocks) return ZC_E_CUDA;
    const uint32_t row_bytes = cache->format == ZC_FMT_FP4_E2M1 ? cache->head_dim / 2 : cache->head_dim;
    const uint64_t rows = std::max<uint64_t>(1, cache->n_pages * cache->kv_heads * cache->page_tokens);
    CUtensorMap maps[2];
    for (int side = 0; side < 2; ++side)                         // without pages nothing is read, but the descriptor wants an address
        if (!make_cache_map(&maps[side], cache->n_pages ? P.C.elems[side] : P.workspace, rows, row_bytes, std::min(cache->page_tokens, row_bytes == 128 ? 32u : 64u))) return ZC_E_CUDA;
    auto run = [&](auto fp4, auto dim) {
        using One = StreamShape<decltype(fp4)::value, decltype(dim)::value, 1>;
        using Two = StreamShape<decltype(fp4)::value, decltype(dim)::value, 2>;
        using Many = PromptShape<decltype(fp4)::value, decltype(dim)::value>;
        cudaStream_t st = (cudaStream_t)cuda_stream;
        const uint64_t columns = (uint64_t)P.group * std::max(1u, batch->max_new);
        if (columns <= 8) return launch_stream<One>(P, maps[0], maps[1], blocks, st);
        const uint32_t few = few_columns(cache);
        if (columns <= few) return launch_stream<Two>(P, maps[0], maps[1], blocks, st);
        // a sequence alone has the rows that are expected; of several some may have few
        if (batch->n_seqs > 1) P.most_rows = few / P.group;
        if (const cudaError_t e = launch_prompt<Many>(P, blocks, st)) return e;
        return batch->n_seqs > 1 && P.most_rows ? launch_stream<Two>(P, maps[0], maps[1], blocks, st) : cudaSuccess;
    };
    auto dims = [&](auto fp4) {
        return cache->head_dim == 128 ? run(fp4, std::integral_constant<uint32_t, 128>()) : run(fp4, std::integral_constant<uint32_t, 64>());
    };
    return (cache->format == ZC_FMT_FP4_E2M1 ? dims(std::true_type()) : dims(std::false_type())) == cudaSuccess ? ZC_OK : ZC_E_CUDA;
}

}  // extern "C"
