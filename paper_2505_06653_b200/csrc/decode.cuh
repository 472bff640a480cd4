// Codes to bf16 operands (Eq. 3, rounded to nearest even: bit for bit what bof4_dequantize writes), in two ways that use
// different units of an SM, and the warp-wide product of sixteen rows with a few tokens that is built on them.
#pragma once

#include "common.cuh"

namespace bof4 {

// Through a table of level pairs in shared memory, [byte][lane], 256 x 32 x 8 bytes.  Eight codes (even element in the high nibble of its byte) to eight bf16 values (Eq. 3, round to nearest even).
__device__ __forceinline__ void tc_lookup8(uint32_t w, float2 mm, uint32_t pairs, uint32_t lane8, uint32_t* o)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        // byte * 256 + lane * 8 in one permute
        const uint32_t off = __byte_perm(w, lane8, 0x5504u | ((uint32_t)k << 4));
        float2 l;
        asm("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(l.x), "=f"(l.y) : "r"(pairs + off));
        const float2 v = __fmul2_rn(mm, l);
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[k]) : "f"(v.y), "f"(v.x));
    }
}

// Eight products by byte permutes.  lo[0..1], hi[0..1]: bytes of entries 0 ... 7, lo[2..3], hi[2..3]: of 8 ... 15.
__device__ __forceinline__ void lt_lookup8(uint32_t w, const uint32_t (&lo)[4], const uint32_t (&hi)[4], uint32_t* o)
{
    // bits 0 ... 2 of each code select within eight entries; bit 3 selects between the two results of a byte
    uint32_t s = w & 0x77777777u, t = ((w >> 1) & 0x44444444u) | 0x32103210u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        // result bytes: elements 1, 0, 3, 2 (the even element of a byte is its high nibble)
        const uint32_t l = __byte_perm(__byte_perm(lo[0], lo[1], s), __byte_perm(lo[2], lo[3], s), t);
        const uint32_t u = __byte_perm(__byte_perm(hi[0], hi[1], s), __byte_perm(hi[2], hi[3], s), t);
        o[2 * h] = __byte_perm(l, u, 0x4051);
        o[2 * h + 1] = __byte_perm(l, u, 0x6273);
        s >>= 16, t >>= 16;
    }
}
// The 16 products m * level, rounded to bf16, as planes of bytes.
__device__ __forceinline__ void lt_table(float m, const float2* levels, uint32_t (&lo)[4], uint32_t (&hi)[4])
{
    uint32_t p[8];
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        const float4 l = reinterpret_cast<const float4*>(levels)[k / 2];
        const float2 a = __fmul2_rn(make_float2(m, m), make_float2(l.x, l.y)), b = __fmul2_rn(make_float2(m, m), make_float2(l.z, l.w));
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p[k]) : "f"(a.y), "f"(a.x));
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p[k + 1]) : "f"(b.y), "f"(b.x));
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        lo[k] = __byte_perm(p[2 * k], p[2 * k + 1], 0x6420);
        hi[k] = __byte_perm(p[2 * k], p[2 * k + 1], 0x7531);
    }
}

constexpr int kPairBytes = 256 * 32 * 8;

// Fills the table of level pairs; all threads of the CTA (whole warps) take part.
__device__ __forceinline__ void fill_pairs(float2* pairs, const float* __restrict__ levels, int tid, int threads)
{
    const float mine = __ldg(levels + (tid & 15));  // level l sits in the lanes with (lane & 15) == l
#pragma unroll 4
    for (int e = tid; e < 256 * 32; e += threads) {
        const int byte = e >> 5;
        pairs[e] = make_float2(__shfl_sync(kFull, mine, byte >> 4), __shfl_sync(kFull, mine, byte & 15));
    }
}

// ---------------------------------------------------------------- sixteen rows times a few tokens
//
// One warp, 16 rows of the matrix by a stripe of 256 columns, on mma.sync (m16n8k16, bf16, fp32 sums): with one to sixteen tokens
// a product is bound by its codes, and the operand fragments of this instruction can be decoded straight into registers.
// The columns of a product may be taken in any order as long as both operands agree, so lane (g, q) = (lane / 4, lane % 4)
// takes 64 consecutive columns, 64 q ... 64 q + 63 of the stripe, of rows g and 8 + g: 32 code bytes per row, whose eight
// words give the row's part of A for two instructions each, one block constant per row (two for blocks of 32), and of B the
// 64 values of token g, which stay in 32 registers for as many rows as the warp visits.
//
// Decoding is what an SM has to do most here: HBM delivers 43 codes per clock and SM.  Row g goes through the table in
// shared memory (4 bytes of its data path per code: 32 codes per clock at most), row 8 + g through byte permutes (2.8 instructions
// of the integer pipe per code: 23 per clock); together they could take 39.

constexpr int kFewStripe = 256;

struct FewCodes {
    uint4 v[4];  // row g: 64 codes, row 8 + g: 64 codes
};
// a, b: the lane's first byte in rows g and 8 + g; live0, live1: the lane's first and last 32 columns exist (and the row does)
__device__ __forceinline__ void few_load(FewCodes& c, const uint8_t* a, const uint8_t* b, bool a0, bool a1, bool b0, bool b1)
{
    const uint8_t* p[4] = {a, a + 16, b, b + 16};
    const bool live[4] = {a0, a1, b0, b1};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        c.v[k] = make_uint4(0u, 0u, 0u, 0u);
        if (live[k])
            asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(c.v[k].x), "=r"(c.v[k].y), "=r"(c.v[k].z), "=r"(c.v[k].w)
                         : "l"(p[k]));
    }
}
template <class ST>
__device__ __forceinline__ float few_scale(const void* scales, int64_t b, bool live);
template <>
__device__ __forceinline__ float few_scale<F32>(const void* scales, int64_t b, bool live)
{
    return live ? __ldg(static_cast<const float*>(scales) + b) : 0.0f;
}
template <>
__device__ __forceinline__ float few_scale<BF16>(const void* scales, int64_t b, bool live)
{
    return live ? __uint_as_float((uint32_t)__ldg(static_cast<const uint16_t*>(scales) + b) << 16) : 0.0f;
}
// The 64 values of a token from the lane's first column, as 32 pairs.
__device__ __forceinline__ void few_tokens(uint32_t (&x)[32], const uint16_t* p, bool live0, bool live1)
{
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint4 u = (k < 4 ? live0 : live1) ? *(reinterpret_cast<const uint4*>(p) + k) : make_uint4(0u, 0u, 0u, 0u);
        x[4 * k] = u.x, x[4 * k + 1] = u.y, x[4 * k + 2] = u.z, x[4 * k + 3] = u.w;
    }
}
__device__ __forceinline__ void few_mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// acc[n]: rows g (0, 1) and 8 + g (2, 3), tokens 8 n + 2 q and 8 n + 2 q + 1.  m: constants of row g, of row 8 + g; with
// HALF those of their first 32 columns in m[0], m[2] and of the last 32 in m[1], m[3].
template <bool HALF, int NT>
__device__ __forceinline__ void few_multiply(const FewCodes& c, const float (&m)[4], const uint32_t (&x)[NT][32], float (&acc)[NT][4],
                                             uint32_t pairs, uint32_t lane8, const float2* levels)
{
    uint32_t lo[4], hi[4];
    lt_table(m[2], levels, lo, hi);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (HALF && j == 4) lt_table(m[3], levels, lo, hi);
        const uint4 va = c.v[j >> 2], vb = c.v[2 + (j >> 2)];
        const uint32_t wa = (j & 3) == 0 ? va.x : (j & 3) == 1 ? va.y : (j & 3) == 2 ? va.z : va.w;
        const uint32_t wb = (j & 3) == 0 ? vb.x : (j & 3) == 1 ? vb.y : (j & 3) == 2 ? vb.z : vb.w;
        const float ma = HALF && j >= 4 ? m[1] : m[0];
        uint32_t a[4], b[4];
        tc_lookup8(wa, make_float2(ma, ma), pairs, lane8, a);
        lt_lookup8(wb, lo, hi, b);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int n = 0; n < NT; ++n) few_mma(acc[n], a[2 * h], b[2 * h], a[2 * h + 1], b[2 * h + 1], x[n][4 * j + 2 * h], x[n][4 * j + 2 * h + 1]);
    }
}

}  // namespace bof4
