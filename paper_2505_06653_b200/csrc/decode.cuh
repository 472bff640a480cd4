// Codes to bf16 operands (Eq. 3, rounded to nearest even: bit for bit what bof4_dequantize writes), in two ways that use
// different units of an SM, and the warp-wide product of sixteen rows with a few tokens that is built on them.
#pragma once

#include "tc.cuh"

namespace bof4 {

// Through a table of level pairs in shared memory, [byte][lane], 256 x 32 x 8 bytes.  Eight codes (even element in the high nibble of
// its byte) to eight bf16 values (Eq. 3, round to nearest even).
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

// The instruction itself: the intrinsic masks a selector that is not a constant, at the price of another instruction each time.
__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t s)
{
    uint32_t r;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(s));
    return r;
}
// Eight products by byte permutes.  lo[0..1], hi[0..1]: bytes of entries 0 ... 7, lo[2..3], hi[2..3]: of 8 ... 15.
__device__ __forceinline__ void lt_lookup8(uint32_t w, const uint32_t (&lo)[4], const uint32_t (&hi)[4], uint32_t* o)
{
    // bits 0 ... 2 of each code select within eight entries; bit 3 selects between the two results of a byte
    uint32_t s = w & 0x77777777u, t = ((w >> 1) & 0x44444444u) | 0x32103210u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        // result bytes: elements 1, 0, 3, 2 (the even element of a byte is its high nibble)
        const uint32_t l = prmt(prmt(lo[0], lo[1], s), prmt(lo[2], lo[3], s), t);
        const uint32_t u = prmt(prmt(hi[0], hi[1], s), prmt(hi[2], hi[3], s), t);
        o[2 * h] = prmt(l, u, 0x4051);
        o[2 * h + 1] = prmt(l, u, 0x6273);
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

constexpr int kPairBytes = 256 * 32 * 8;  // level pairs per code byte, a column per lane

// Fills the table of level pairs; all warps of the CTA take part.  A row of the table is the same pair 32 times: a warp
// writes rows in turn, the levels in its registers.
__device__ __forceinline__ void fill_pairs(float2* pairs, const float* __restrict__ levels, int tid, int threads)
{
    float lv[16];
#pragma unroll
    for (int l = 0; l < 16; l += 4) {
        const float4 v = make_float4(__ldg(levels + l), __ldg(levels + l + 1), __ldg(levels + l + 2), __ldg(levels + l + 3));
        lv[l] = v.x, lv[l + 1] = v.y, lv[l + 2] = v.z, lv[l + 3] = v.w;
    }
    for (int hi = tid >> 5; hi < 16; hi += threads >> 5) {
        float h = lv[15];
#pragma unroll
        for (int l = 14; l >= 0; --l) h = hi == l ? lv[l] : h;
        float2* const row = pairs + hi * (16 * 32) + (tid & 31);
#pragma unroll
        for (int l = 0; l < 16; ++l) row[l * 32] = make_float2(h, lv[l]);
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
// Decoding is what an SM has to do most here: HBM delivers 43 codes per clock and SM.  The table in shared memory takes 4
// bytes of its data path per code (32 codes per clock at most) and one instruction of the integer pipe, byte permutes take 2.9 of
// that pipe (22 per clock).  Three quarters of the codes go through the table, the last 32 columns of row 8 + g
// through permutes: 42 per clock for the one, 40 for the other.  Together with the conversions (each code one half), addresses and
// products an SM reaches 18 to 20 (28672 x 8192 by one token 42 us: shared memory 64 %, integer pipe 66 %, issue 60 %).

constexpr int kFewStripe = 256;

struct FewCodes {
    uint4 v[4];  // row g: 64 codes, row 8 + g: 64 codes
};
// Codes travel to shared memory by TMA, kFewAhead units ahead, into a ring that the warp owns: one lane requests a unit (16 rows of 128
// bytes, in the 128-byte swizzle, zeros outside the matrix), and every lane reads the 32 bytes of its columns from rows g and
// 8 + g without meeting a bank twice.  Loads and addresses of the lanes' own took 40 % of the instructions of a unit.
constexpr int kFewUnit = 2048, kFewAhead = 2, kFewSlots = kFewAhead + 1;
__device__ __forceinline__ void few_read(FewCodes& c, uint32_t slot, int lane)
{
    const uint32_t g = (uint32_t)lane >> 2, q = (uint32_t)lane & 3u;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(c.v[k].x), "=r"(c.v[k].y), "=r"(c.v[k].z), "=r"(c.v[k].w)
                     : "r"(slot + (g + 8u * (k >> 1)) * 128u + ((2u * q + (k & 1u)) ^ g) * 16u)
                     : "memory");
}
// The lane's block constants of a unit as they are in memory, widened where they are used so that nothing waits for the loads
// before: row g in [0] (with HALF its first 32 columns in [0], its last in [1]), row 8 + g in [2], [3].  a, b: the constants of
// the lane's first weights in the two rows; live: bits 0, 1: row g and the lane's first and last 32 columns exist, 2, 3: row 8 + g.
template <class ST, bool HALF>
struct FewConst {
    uint32_t v[4];
    __device__ __forceinline__ void load(const void* scales, int64_t a, int64_t b, uint32_t live)
    {
#pragma unroll
        for (int k = 0; k < 4; k += HALF ? 1 : 2) {
            const int64_t i = (k < 2 ? a : b) + (k & 1);
            v[k] = 0u;
            if (live >> k & 1u) {
                if (ST::code == BOF4_F32) {
                    asm volatile("ld.global.nc.u32 %0, [%1];" : "=r"(v[k]) : "l"(static_cast<const uint32_t*>(scales) + i));
                } else {
                    uint16_t h;
                    asm volatile("ld.global.nc.u16 %0, [%1];" : "=h"(h) : "l"(static_cast<const uint16_t*>(scales) + i));
                    v[k] = h;
                }
            }
        }
    }
    __device__ __forceinline__ float value(int k) const { return __uint_as_float(ST::code == BOF4_F32 ? v[k] : v[k] << 16); }
};
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
// The table of level pairs lies at this address of shared memory, so that one permute makes a whole address of a code byte and the
// lane: byte * 256 + lane * 8 + 0x10000.  What comes before it is the kernel's to use, the ring lies behind it.
constexpr uint32_t kFewTable = 0x10000u, kFewRing = kFewTable + kPairBytes;
// Eight codes through the table, in two halves: the look-ups, and products and rounding.  column = lane * 8 + kFewTable.
__device__ __forceinline__ void few_fetch8(uint32_t w, uint32_t column, float2 (&l)[4])
{
#pragma unroll
    for (int k = 0; k < 4; ++k)
        asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(l[k].x), "=f"(l[k].y) : "r"(__byte_perm(w, column, 0x7604u | ((uint32_t)k << 4))));
}
__device__ __forceinline__ void few_round8(float m, const float2 (&l)[4], uint32_t (&o)[4])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 v = __fmul2_rn(make_float2(m, m), l[k]);
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[k]) : "f"(v.y), "f"(v.x));
    }
}
__device__ __forceinline__ uint32_t few_word(const uint4& v, int j) { return j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w; }

// acc[n]: rows g (0, 1) and 8 + g (2, 3), tokens 8 n + 2 q and 8 n + 2 q + 1.  A step is a word of each row; the look-ups of the
// next step are issued before the products of this one.
template <class ST, bool HALF, int NT>
__device__ __forceinline__ void few_multiply(const FewCodes& c, const FewConst<ST, HALF>& raw, const uint32_t (&x)[NT][32], float (&acc)[NT][4],
                                             uint32_t column, const float2* levels)
{
    const float m[4] = {raw.value(0), HALF ? raw.value(1) : raw.value(0), raw.value(2), HALF ? raw.value(3) : raw.value(2)};
    uint32_t lo[4], hi[4];
    lt_table(m[3], levels, lo, hi);
    float more[NT][4] = {};  // a second chain of sums
    float2 la[2][4], lb[2][4];
    // step i takes words of the first and of the last 32 columns in turn: table and permutes next to one another
    auto word = [](int i) { return (i & 1) * 4 + (i >> 1); };
    auto fetch = [&](int i) {
        const int j = word(i);
        few_fetch8(few_word(c.v[j >> 2], j & 3), column, la[i & 1]);
        if (j < 4) few_fetch8(few_word(c.v[2 + (j >> 2)], j & 3), column, lb[i & 1]);
    };
    fetch(0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int j = word(i);
        if (i < 7) fetch(i + 1);
        uint32_t a[4], b[4];
        few_round8(m[j >> 2], la[i & 1], a);
        if (j < 4) few_round8(m[2], lb[i & 1], b);
        else lt_lookup8(few_word(c.v[2 + (j >> 2)], j & 3), lo, hi, b);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int n = 0; n < NT; ++n)
                few_mma(j < 4 ? acc[n] : more[n], a[2 * h], b[2 * h], a[2 * h + 1], b[2 * h + 1], x[n][4 * j + 2 * h], x[n][4 * j + 2 * h + 1]);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[n][k] += more[n][k];
}

}  // namespace bof4
