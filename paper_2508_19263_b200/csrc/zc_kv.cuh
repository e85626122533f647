// What the kernels on a quantised key/value cache share: descriptors, places of tokens, conversions, argument checks.
#pragma once
#include "zc_fp8.cuh"

namespace zc {

constexpr uint32_t kKvBlock = 32;                         // elements that share a scale byte
constexpr uint32_t kKvGaveUp = 1, kKvCorrupt = 2;         // what kernels leave for zc_kv_status

unsigned int* kv_marks_word();                            // on the current device; null on an error

struct KvCache {
    uint8_t *elems[2], *scales[2];                        // keys, values
    uint32_t n_pages, page_shift, heads;
};
struct KvBatch {
    const int32_t *table, *lens, *first;
    uint64_t ld_table;
    uint32_t max_pages, n_seqs, n_rows, capacity;         // capacity: tokens that a table's row has room for
    unsigned int* marks;
};
struct KvTensor {
    uint8_t* d;
    uint64_t ld_row, ld_head;                             // bytes
};

// Length of a sequence, within what its row of the table has room for.
__device__ __forceinline__ int kv_len(const KvBatch& B, uint32_t b)
{
    const int n = B.lens[b];
    if (n >= 0 && (uint32_t)n <= B.capacity) return n;
    atomicOr(B.marks, kKvCorrupt);
    return n < 0 ? 0 : (int)B.capacity;
}
// Page of a place of a sequence; -1 for one outside the cache.
__device__ __forceinline__ int kv_page(const KvCache& C, const KvBatch& B, uint32_t b, uint32_t place)
{
    const int p = B.table[(uint64_t)b * B.ld_table + place];
    if ((uint32_t)p < C.n_pages) return p;
    atomicOr(B.marks, kKvCorrupt);
    return -1;
}
// The last sequence whose rows begin at or before `row`, -1 if there is none.  All lanes of a warp together, 32 ways at a time.
__device__ __forceinline__ int kv_find(const KvBatch& B, int row)
{
    const uint32_t lane = threadIdx.x & 31;
    uint32_t lo = 0, n = B.n_seqs;
    bool any = false;
    while (true) {
        const uint32_t step = (n + 31) / 32, at = lane * step;
        const uint32_t hit = __ballot_sync(0xFFFFFFFFu, at < n && B.first[lo + at] <= row);
        if (hit == 0) return any ? (int)lo : -1;
        any = true;
        const uint32_t k = 31 - __clz(hit);
        lo += k * step;
        n = min(step, n - k * step);
        if (step == 1) return (int)lo;
    }
}
// Sequence and position of a row, from a sequence at or before its own; false: the row is nobody's, or its position negative.
__device__ __forceinline__ bool kv_position(const KvBatch& B, int row, uint32_t& b, int& pos)
{
    while (b + 1 < B.n_seqs && B.first[b + 1] <= row) ++b;
    const int from = B.first[b], to = B.first[b + 1];
    if (row < from || row >= to) { pos = -1; return false; }
    const long long at = (long long)kv_len(B, b) - ((long long)to - from) + ((long long)row - from);
    pos = (int)max(at, -1ll);
    return true;
}

// Elements of 32 bits of a cache's word: 8 in FP4, 4 in E4M3, as pairs of FP16, two neighbours a pair.
__device__ __forceinline__ void fp4_to_half(uint32_t w, uint32_t h[4])
{
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\tcvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}
__device__ __forceinline__ void e4m3_to_half(uint32_t w, uint32_t h[2])
{
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(h[0]), "=r"(h[1]) : "r"(w));
}
__device__ __forceinline__ float2 half_pair(uint32_t h) { return __half22float2(*reinterpret_cast<const __half2*>(&h)); }
// 2^(s - 127); NaN for 255
__device__ __forceinline__ float e8m0_value(uint32_t s) { return __uint_as_float(s == 255 ? 0x7FFFFFFFu : max(s << 23, 0x00400000u)); }

// ---- host ----
inline zc_status check_cache(const zc_kv_cache* c)
{
    if (!c) return ZC_E_INVALID_ARG;
    if (c->format != ZC_FMT_FP4_E2M1 && c->format != ZC_FMT_FP8_E4M3) return ZC_E_UNSUPPORTED;
    if (c->head_dim != 64 && c->head_dim != 128) return ZC_E_UNSUPPORTED;
    if (c->page_tokens < 16 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1))) return ZC_E_UNSUPPORTED;
    if (c->kv_heads == 0) return ZC_E_INVALID_ARG;
    if (c->kv_heads > ZC_KV_MAX_HEADS || c->n_pages >= (1ull << 31) || c->n_pages * c->kv_heads * c->page_tokens >= (1ull << 31)) return ZC_E_TOO_LARGE;
    for (const void* p : {c->d_k_elems, c->d_k_scales, c->d_v_elems, c->d_v_scales})
        if (!aligned16(p) || (!p && c->n_pages)) return ZC_E_INVALID_ARG;
    return ZC_OK;
}
inline zc_status check_batch(const zc_kv_cache* c, const zc_kv_batch* b)
{
    if (!b) return ZC_E_INVALID_ARG;
    if (b->n_seqs > ZC_KV_MAX_SEQS || b->n_rows >= kMaxDim || (uint64_t)b->max_pages * c->page_tokens >= (1ull << 31)) return ZC_E_TOO_LARGE;
    if (b->n_seqs == 0 || b->n_rows == 0) return ZC_OK;                     // nothing is read or written
    if (!b->d_lens || !b->d_first || (!b->d_page_table && b->max_pages) || b->ld_page_table < b->max_pages || b->ld_page_table >= (1ull << 39)) return ZC_E_INVALID_ARG;
    for (const void* p : {b->d_page_table, b->d_lens, b->d_first})
        if (reinterpret_cast<uintptr_t>(p) % 4) return ZC_E_INVALID_ARG;
    return ZC_OK;
}
inline zc_status check_tensor(const zc_kv_tensor* t, uint32_t width, uint64_t rows, uint32_t heads, uint32_t dim)
{
    if (!t || !t->d || reinterpret_cast<uintptr_t>(t->d) % width) return ZC_E_INVALID_ARG;
    if ((rows > 1 && t->ld_row < dim) || (heads > 1 && t->ld_head < dim) || t->ld_row >= (1ull << 39) || t->ld_head >= (1ull << 39)) return ZC_E_INVALID_ARG;
    return ZC_OK;
}
inline KvCache device_cache(const zc_kv_cache* c)
{
    KvCache d{};
    d.elems[0] = (uint8_t*)c->d_k_elems;
    d.elems[1] = (uint8_t*)c->d_v_elems;
    d.scales[0] = (uint8_t*)c->d_k_scales;
    d.scales[1] = (uint8_t*)c->d_v_scales;
    d.n_pages = (uint32_t)c->n_pages;
    d.heads = c->kv_heads;
    while ((1u << d.page_shift) < c->page_tokens) ++d.page_shift;
    return d;
}
inline KvBatch device_batch(const zc_kv_cache* c, const zc_kv_batch* b, unsigned int* marks)
{
    KvBatch d{};
    d.table = b->d_page_table;
    d.lens = b->d_lens;
    d.first = b->d_first;
    d.ld_table = b->ld_page_table;
    d.max_pages = b->max_pages;
    d.n_seqs = b->n_seqs;
    d.n_rows = (uint32_t)b->n_rows;
    d.capacity = b->max_pages * c->page_tokens;
    d.marks = marks;
    return d;
}
inline KvTensor device_tensor(const zc_kv_tensor* t, uint32_t width)
{
    return t ? KvTensor{(uint8_t*)t->d, t->ld_row * width, t->ld_head * width} : KvTensor{};
}

}  // namespace zc
