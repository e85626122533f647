// What the kernels on FP8 matrices share: number formats, wide loads, and the PTX of clusters, tensor copies and the
// fifth-generation tensor cores.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "zc_device.cuh"

namespace zc {

constexpr uint32_t kScaleCols = 128;          // columns that share a scale byte
constexpr uint64_t kMaxDim = 1ull << 31;      // rows and columns stay below (tensor copies take 32-bit signed coordinates)

inline uint64_t ceil_div(uint64_t a, uint64_t b) { return a / b + (a % b != 0); }

inline bool fp8_format(uint32_t f) { return f == ZC_FMT_FP8_E4M3 || f == ZC_FMT_FP8_E5M2; }
inline uint32_t real_bytes(uint32_t t) { return t == ZC_REAL_F32 ? 4u : (t == ZC_REAL_BF16 || t == ZC_REAL_F16) ? 2u : 0u; }

// Arguments that every operator checks alike.  Elements are read and written in 16-byte pieces and by tensor copies, so
// rows begin on 16-byte boundaries; scale bytes have no alignment.
inline zc_status check_matrix(const zc_fp8_matrix* m)
{
    if (!m) return ZC_E_INVALID_ARG;
    if (!fp8_format(m->format)) return ZC_E_UNSUPPORTED;
    if (m->block_rows != 1 && m->block_rows != 128) return ZC_E_UNSUPPORTED;
    if (m->rows >= kMaxDim || m->cols >= kMaxDim) return ZC_E_TOO_LARGE;
    if (!m->rows || !m->cols) return ZC_OK;                  // nothing of it is read or written
    if (!m->d_elems || !m->d_scales) return ZC_E_INVALID_ARG;
    if (!aligned16(m->d_elems) || m->ld_elems % 16 || m->ld_elems < m->cols || m->ld_elems >= (1ull << 39)) return ZC_E_INVALID_ARG;
    if (m->ld_scales < ceil_div(m->cols, kScaleCols) || m->ld_scales >= (1ull << 39)) return ZC_E_INVALID_ARG;
    return ZC_OK;
}

unsigned int* moe_marks_word();                           // what the kernels of zc_fp8_moe left for zc_fp8_status

__device__ __forceinline__ float finite_abs(float v)
{
    const float a = fabsf(v);
    return a < __int_as_float(0x7F800000) ? a : 0.0f;        // NaN compares false as well
}

// Scale byte of a block: e + 127.
template <bool E5M2>
__device__ __forceinline__ uint32_t scale_byte(float amax)
{
    const uint32_t b = __float_as_uint(amax);
    const int e = (int)(b >> 23) - 127 - (E5M2 ? 15 : 8) + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return b == 0 || e < -127 ? 0u : (uint32_t)(e + 127);    // e <= 128 - 8: no clamp above
}
__device__ __forceinline__ float inverse_scale(uint32_t s) { return __uint_as_float((254u - s) << 23); }   // 2^-(s-127), s <= 247


__device__ __forceinline__ void sts128(uint32_t addr, const uint32_t v[4])
{
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" :: "r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
// ---- 32-byte global accesses (one sector per lane); 32-byte aligned ----
__device__ __forceinline__ void ld_v8(const void* p, uint32_t v[8])
{
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "l"(p));
}
__device__ __forceinline__ uint4 ld_stream_v4(const void* p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// 16 bytes to shared memory past the registers, of which the first `have` are read and the others become zeros
__device__ __forceinline__ void async_copy16(uint32_t to, const void* from, uint32_t have)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(to), "l"(from), "r"(have) : "memory");
}
__device__ __forceinline__ void async_copy_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ uint4 lds128(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}

// ---- programmatic dependent launch ----
// A kernel may be on the GPU, and set up its barriers and tensor memory, while the one before it in the stream ends; it
// touches nothing that other kernels read or write before grid_wait(), which waits for all of them.  It lets the next one in
// only after that, so that no more than two of a stream's kernels are there at a time and what the next one reads is not still
// being read, and cached, by the one before this.  What it reads may have been written while it was there already, so its loads are
// the ordinary ones, never those (`.nc`, __ldg) that take the memory to be unchanged for as long as the kernel is there.
inline cudaLaunchAttribute launch_early()
{
    cudaLaunchAttribute a{};
    a.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    a.val.programmaticStreamSerializationAllowed = 1;
    return a;
}
__device__ __forceinline__ void grid_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// ---- warps ----
// One lane of a converged warp.  Copies, matrix instructions and commits take their operands from uniform registers: in a loop
// that the whole warp goes through, with the one lane chosen at each of them, the operands are there; in a loop that only lane 0
// goes through each of them is moved there first (8192 x 14336 x 4096 in short runs: 447 us, 388 so).
__device__ __forceinline__ bool elect_one()
{
    uint32_t is;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
    return is != 0;
}
__device__ __forceinline__ uint32_t warp_index() { return __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0); }

// ---- clusters ----
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait()
{
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_sync()
{
    cluster_arrive();
    cluster_wait();
}
// the same place in the shared memory of the cluster's block `rank`
__device__ __forceinline__ uint32_t map_shared(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}

// ---- mbarriers by shared address, across a cluster ----
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
// bytes that nobody will copy count as copied
__device__ __forceinline__ void bar_forgo(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
// Ordered within the block only.  At the cluster's scope every arrival waits for the thread's earlier writes and every wait
// drops the L1: 0.8 us a step of the mixture-of-experts kernels instead of 0.4.
__device__ __forceinline__ void bar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ void bar_arrive_cluster(uint32_t cluster_bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" :: "r"(cluster_bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}

// the same wait for what another block of the cluster wrote before it arrived
__device__ __forceinline__ bool bar_try_cluster(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}

// ---- tensor copies global -> shared; the barrier may be another block's of the pair (GROUP 2) ----
template <int GROUP>
__device__ __forceinline__ void tensor_copy(uint32_t dst, const void* map, int x, int y, uint32_t bar)
{
    if (GROUP == 1)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];"
                     :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// the way back; one thread's copies are committed as a group
__device__ __forceinline__ void tensor_store(const void* map, int x, int y, uint32_t src)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];\n\tcp.async.bulk.commit_group;"
                 :: "l"(map), "r"(x), "r"(y), "r"(src) : "memory");
}
// at most N of the thread's groups have not been read out of shared memory yet
template <int N>
__device__ __forceinline__ void tensor_store_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" :: "n"(N) : "memory"); }
__device__ __forceinline__ void prefetch_map(const void* map)
{
    asm volatile("prefetch.tensormap [%0];" :: "l"(map) : "memory");
}

// ---- tensor memory and tensor cores ----
template <int GROUP>
__device__ __forceinline__ void tmem_alloc(uint32_t where, uint32_t cols)
{
    if (GROUP == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(where), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(where), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
}
template <int GROUP>
__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t cols)
{
    if (GROUP == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(base), "r"(cols));
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(base), "r"(cols));
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// D[128 or 256 x N] (+)= A B^T of one step of 32 columns; FP8 operands in shared memory, a scale byte per row of A and of B
// in tensor memory (kind::mxf8f6f4: products times 2^(sa+sb-254), accumulated in FP32)
template <int GROUP>
__device__ __forceinline__ void mma_scaled(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t add)
{
    if (GROUP == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(add) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(add) : "memory");
}
// the barrier (in every block of the group) completes when all matrix instructions issued so far have
template <int GROUP>
__device__ __forceinline__ void mma_commit(uint32_t bar)
{
    if (GROUP == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     :: "r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t v[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
                   "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
                   "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
                   "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
                 : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
// eight columns of a quarter's 32 lanes; not complete before tmem_ld_wait
__device__ __forceinline__ void tmem_ld8(uint32_t addr, float v[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]) : "r"(addr));
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// 512 bytes of scale words, [32][4] in shared memory, to four columns of every quarter of tensor memory (in every block of the
// group, from its own shared memory): word (i, j) is that of row 32 j + i
template <int GROUP>
__device__ __forceinline__ void tmem_copy_scales(uint32_t addr, uint32_t shared)
{
    // no swizzle, groups of eight 16-byte rows 128 bytes apart
    const uint64_t desc = (uint64_t)((shared & 0x3FFFFu) >> 4) | (1ull << 16) | ((uint64_t)(128 >> 4) << 32) | (1ull << 46);
    if (GROUP == 1) asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" :: "r"(addr), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" :: "r"(addr), "l"(desc) : "memory");
}
// shared memory written by ordinary stores becomes visible to tensor copies and matrix instructions
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Operand tile in shared memory: rows of 128 bytes in the 128-byte swizzle, groups of 8 rows 1024 bytes apart
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr)
{
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

// ---- warp-wide matrix instruction (few-token kernels, where the bytes of the weights bound the time) ----
__device__ __forceinline__ void mma_bf16(float c[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float c[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

}  // namespace zc
