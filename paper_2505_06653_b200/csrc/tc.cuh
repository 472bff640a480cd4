// Pieces shared by the kernels that multiply on the tensor cores (gemm_tc.cu, linear_tc.cu): matrix descriptors, bounded
// waits, TMA loads, tensor-memory reads, tickets of cut tiles.
#pragma once

#include <atomic>
#include <chrono>

#include <cuda.h>

#include "common.cuh"

namespace bof4 {

constexpr uint32_t kTcSpinLimit = 1u << 16;      // try_wait calls before a wait gives up (a k-block takes microseconds)

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// Shared-memory matrix descriptor of a K-major tile in the 128-byte swizzled layout: start
// address and offsets in units of 16 bytes, leading offset 1 (unused for swizzled K-major), stride
// between 8-row groups 1024 bytes, descriptor version 1, layout type 2 (128-byte swizzle).
// `leading` in bytes: for an M-major tile the stride between groups of 64 of M (the stride is then between groups of 8 of K).
__device__ __forceinline__ uint64_t tc_smem_desc(uint32_t addr, uint32_t leading = 16)
{
    uint64_t d = 0;
    d |= (uint64_t)((addr >> 4) & 0x3fffu);
    d |= (uint64_t)(leading >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}

__device__ __forceinline__ bool tc_wait(uint32_t bar, uint32_t parity)
{
    for (uint32_t it = 0; it < kTcSpinLimit; ++it) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(bar), "r"(parity), "r"(1000u)  // suspended for up to a microsecond instead of polling
            : "memory");
        if (ok) return true;
    }
    return false;
}

// After a wait has run out: copies and tensor-core instructions that were issued before may still be under way.  They take
// microseconds; they get a bounded 100 before shared and tensor memory go away.
__device__ __forceinline__ void tc_settle()
{
    for (int i = 0; i < 100; ++i) __nanosleep(1000);
}

// A look at a barrier, without a wait.
__device__ __forceinline__ bool tc_look(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0u;
}
// One lane of a converged warp, always the same one.
__device__ __forceinline__ bool tc_elect()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0u;
}

// A block constant as it is in memory; widened where it is used, so that nothing waits for the load before.
template <class ST>
struct TcConst;
template <>
struct TcConst<F32> {
    float v;
    __device__ __forceinline__ void load(const void* scales, int64_t b)
    {
        asm volatile("ld.global.nc.f32 %0, [%1];" : "=f"(v) : "l"(static_cast<const float*>(scales) + b));
    }
    __device__ __forceinline__ float value() const { return v; }
};
template <>
struct TcConst<BF16> {
    uint16_t v;
    __device__ __forceinline__ void load(const void* scales, int64_t b)
    {
        asm volatile("ld.global.nc.u16 %0, [%1];" : "=h"(v) : "l"(static_cast<const uint16_t*>(scales) + b));
    }
    __device__ __forceinline__ float value() const { return __uint_as_float((uint32_t)v << 16); }
};

__device__ __forceinline__ void tc_arrive(unsigned long long* bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tc_load_box(uint32_t dst, const CUtensorMap* map, unsigned long long* bar, uint32_t bytes, int x, int y)
{
    const uint32_t b = smem_u32(bar);
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(b), "r"(bytes) : "memory");
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 :
                 : "r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(b), "r"(x), "r"(y)
                 : "memory");
}

// Eight 32-bit columns of the warp's 32 rows from tensor memory.
__device__ __forceinline__ void tc_load8(uint32_t addr, uint32_t (&v)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
// The tensor-core instructions that the lane with lead = 1 has issued arrive on `bar` when they have completed.
__device__ __forceinline__ void tc_commit(unsigned long long* bar, uint32_t lead)
{
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "setp.ne.b32 q, %1, 0;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar)), "r"(lead)
        : "memory");
}

// A tile's ticket.  The cell needs no preparation: every CTA that has a part of the tile first makes sure that
// it carries the launch's 56-bit epoch (with no arrivals yet), long before it arrives; the last arrival clears it.
__device__ __forceinline__ void tc_ticket_open(unsigned long long* cell, unsigned long long epoch)
{
    unsigned long long old = *reinterpret_cast<volatile unsigned long long*>(cell);
    while ((old & ~255ull) != epoch) {
        const unsigned long long seen = atomicCAS(cell, old, epoch);
        if (seen == old) break;
        old = seen;  // somebody else opened it or arrived: at most `ctas` rounds
    }
}

// ---------------------------------------------------------------- host side

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Tensor map of a row-major matrix of 2-byte (bf16) or 1-byte elements, `pitch` bytes between rows, with a box of `box_bytes`
// (128 or 64) x box_rows and the swizzle of that width: operands land in the layout that the tcgen05 descriptors name, codes
// in one that sixteen-byte reads of neighbouring rows find without bank conflicts.  Elements outside the matrix read as zero.
inline int tc_make_map(const char* who, const void* p, int esize, int64_t cols, int64_t rows, int64_t pitch, int box_bytes, int box_rows,
                       CUtensorMap* map)
{
    static std::atomic<EncodeTiledFn> known{nullptr};
    EncodeTiledFn fn = known.load(std::memory_order_relaxed);
    if (!fn) {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        BOF4_CUDA_TRY(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q));
        if (!f || q != cudaDriverEntryPointSuccess) {
            set_error("%s: the driver does not provide cuTensorMapEncodeTiled", who);
            return BOF4_ERR_CUDA;
        }
        fn = reinterpret_cast<EncodeTiledFn>(f);
        known.store(fn, std::memory_order_relaxed);
    }
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)pitch};
    const cuuint32_t box[2] = {(cuuint32_t)(box_bytes / esize), (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1, 1};
    const CUresult r = fn(map, esize == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims,
                          strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          box_bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        set_error("%s: cuTensorMapEncodeTiled failed with code %d", who, (int)r);
        return BOF4_ERR_CUDA;
    }
    return BOF4_OK;
}

// A name for every launch, no two alike: 56 bits that mix a counter with the time the library was loaded.
inline unsigned long long tc_next_epoch()
{
    static std::atomic<unsigned long long> counter{(unsigned long long)std::chrono::steady_clock::now().time_since_epoch().count()};
    unsigned long long z = counter.fetch_add(1) * 0x9e3779b97f4a7c15ull;  // odd: distinct values stay distinct
    z ^= z >> 29;
    z &= ~255ull;
    return z ? z : 256ull;
}

}  // namespace bof4
