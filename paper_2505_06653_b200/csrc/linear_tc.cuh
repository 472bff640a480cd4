// Products of a 4-bit matrix with any number of tokens on the tensor cores (tcgen05), forward and backward:
//
//   forward   z[t, r] = sum_c W^[r, c] x[t, c]          M = 128 rows r,    K = columns c
//   backward  dx[t, c] = sum_r dz[t, r] W^[r, c]         M = 128 columns c, K = rows r
//
// W^ is the dequantised weight rounded to bf16, bit for bit what bof4_dequantize writes (Eq. 3), with the stored values of
// the outliers in their places; products are exact, sums fp32 in tensor memory.  A tile is 128 of M by up to 256 tokens (N),
// so that a decoded weight is used for up to 256 tokens.
//
// The codes of both directions are decoded row by row as they are stored: a thread takes 64 consecutive codes of one row of
// W, which share a block constant, and writes the 128 bytes of their bf16 values as one row of the A tile.  Forward that row
// is a row of M with 64 of K (a K-major operand), backward it is one of K with 64 of M (an M-major operand): the tile in
// shared memory is the same, only the matrix descriptor and the order in which code bytes are fetched differ.
//
// Decoding.  A thread forms the 16 possible products constant * level of its block once (eight packed multiplications and
// conversions for 64 weights) and keeps them in eight registers, the low bytes of the 16 bf16 values in four and the high
// bytes in four.  A code is then looked up by byte permutes: four codes take two permutes of the lower and the upper eight
// entries and one that picks between them by bit 3, for the low and for the high bytes, and two that put the bytes together.
// That is 2.6 instructions per weight of the integer pipe (3.0 with the making of the table: 390 to 420 cycles per k-block of
// 128 x 64 weights) and no shared memory; a table of level pairs in shared memory (gemm_tc.cu) takes 4 bytes of its data path
// per weight, which the tensor cores need here for their own operands.  Tiles of up to 64 tokens leave both the room and the
// cycles for the table, and half of the codes go through it.
//
// The work is dealt as in gemm_tc.cu: lines (four k-blocks of 64 of K) of all tiles, tile after tile, in equal contiguous
// parts to one CTA per SM; a tile that several CTAs share is summed in their order by the one that completes it last (a
// ticket: nobody waits).  Warps with one job each, coupled by mbarriers:
//
//   16 producers  four groups of four warps, a k-block of the line each, which always go to the same stages.  (Every line has
//                 four k-blocks: groups that skipped some could get two turns of a stage apart, and a barrier's parity
//                 would no longer say which.)
//   1 issuer      four tcgen05.mma (M = 128, N = tokens, K = 16) per k-block, tcgen05.commit hands the stage back
//   1 tokens, 1 codes   TMA loads of the B operand, and of half lines of codes (128 rows of 64 bytes in both directions)
//   4 results     read a finished accumulator (there are two) while the next tile runs
//
// A stage has one barrier that both operands complete, and is handed back by one commit; codes are handed back by half lines,
// so that the ring needs 16 KiB less than whole lines would.
//
// What bounds it (profiles: 28672 x 8192 by 32 tokens, 14336 x 4096 by 2048): up to 64 tokens decoding, about 760 cycles per
// k-block with shared memory and the integer pipe at 68 % each; at 256 tokens the data path of shared memory, through which both
// operands go in and out: 832 cycles per k-block, of which the tensor cores need 512.  28672 x 8192: 24 tokens 84 us, 64 89, 128
// 100, 256 123, 2048 870 (1107 TFLOP/s; the power limit holds the clock down).  Two SMs on one tile (cta_group::2, each decoding
// half of it) took 1.7 times as long: the producers of both wait for one another at every stage.  24 warps leave a thread 80 registers; every
// instantiation spills 5 to 11 more, the gated ones 12 to 15, those whose accumulators take segments 11 to 16.
//
// Every wait is bounded: a time-out sets the status word, everybody leaves, the kernel frees its tensor memory and returns.
#pragma once

#include "decode.cuh"
#include "linear.cuh"
#include "tc.cuh"

namespace bof4 {

constexpr int kLtGroups = 4;                 // producer groups, a k-block of a line and a stage each
constexpr int kLtM = 128, kLtK = 64;
constexpr int kLtMaxN = 256;                 // tokens of a tile; columns of an accumulator
constexpr int kLtABytes = kLtM * kLtK * 2;   // 16 KiB
constexpr int kLtHalfBytes = 8192;           // half a line of codes: two k-blocks; 128 rows x 64 bytes
constexpr int kLtMaxHalves = 8;
constexpr int kLtTableN = 64;                // tokens of a tile up to which there is room, and use, for the table of pairs
constexpr int kLtLongK = 4096;               // K up to which results in fp32 have tiles of any width
constexpr int kLtSegment = 4;                // lines of an accumulator's segment (1024 of K; accumulators that take turns: as many times more)
constexpr int kLtMaxParts = 64;              // of a tile
constexpr int kLtAhead = 6;                  // lines that L2 is asked for before the ring is
constexpr int kLtSmem = 225 * 1024;          // stages and half lines, with slack to align them to 1024 bytes
constexpr int kLtIssue = 16, kLtTokens = 17, kLtCodes = 18, kLtResults = 20;  // warp 19 has no job: the results start at a multiple of 4
constexpr int kLtThreads = 32 * (kLtResults + 4);

struct LtWork {
    int tiles, tiles_n, per_tile;  // tiles, those along the tokens, lines of a tile
    int box_n;                     // tokens of a tile, a multiple of 16
    int k;                         // K
    int halves;                    // half lines of codes in the ring (even, at least four)
    int accs;                      // accumulators of a part of a tile, which the instructions of a k-block use in turn: 4, 2 or 1
    int segment;                   // lines that an accumulator takes at most (SEGMENTS)
    int each, extra;               // lines per CTA, and the remainder
    bool table;                    // half of the codes go through a table
    unsigned long long epoch;
    __host__ __device__ int start(int i) const { return i * each + (i < extra ? i : extra); }
    __device__ int owner(int l) const
    {
        const uint32_t longer = (uint32_t)extra * (uint32_t)(each + 1);
        return (uint32_t)l < longer ? (int)((uint32_t)l / (uint32_t)(each + 1)) : extra + (int)(((uint32_t)l - longer) / (uint32_t)each);
    }
};

__device__ __forceinline__ void lt_load16(uint32_t addr, uint32_t (&v)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(addr));
}
__device__ __forceinline__ void lt_read16(uint32_t addr, uint32_t (&v)[16])  // with the wait, so that no sum can get between the two
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(addr)
        : "memory");
}

// Sums of the segments before, which a lane keeps in the part's slab.  Of a part that others will add to theirs, a lane's row goes to its place, column by column, and each segment is
// added where it lies, without a wait for what is there (nobody else has the place until the part is finished).  Of a tile that the CTA has whole, a warp's four columns of its
// 32 rows lie row by row instead, sixteen bytes a lane (`at`), and are read again with the last segment: columns q ... q + 31, `count` in all.
__device__ __forceinline__ void lt_before(const float* at, int q, int count, float (&z)[32])
{
#pragma unroll
    for (int j = 0; j < 32; j += 4) {
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (at && q + (j & 16) < count) v = __ldcg(reinterpret_cast<const float4*>(at + (q + j) * kLtM));
        z[j] = v.x, z[j + 1] = v.y, z[j + 2] = v.z, z[j + 3] = v.w;
    }
}
template <int N>
__device__ __forceinline__ void lt_put(float* p, const float (&v)[N], bool whole, bool add)
{
    if (whole) {
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            float* const to = p + j * kLtM;
            if (add) asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(to), "f"(v[j]), "f"(v[j + 1]), "f"(v[j + 2]), "f"(v[j + 3]) : "memory");
            else __stcg(reinterpret_cast<float4*>(to), make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]));
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (add) asm volatile("red.relaxed.gpu.global.add.f32 [%0], %1;" ::"l"(p + j * kLtM), "f"(v[j]) : "memory");
            else __stcg(p + j * kLtM, v[j]);
        }
    }
}

__device__ __forceinline__ void lt_read32(uint32_t addr, float (&v)[32])
{
    uint32_t a[16], b[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%32];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%33];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=&r"(a[0]), "=&r"(a[1]), "=&r"(a[2]), "=&r"(a[3]), "=&r"(a[4]), "=&r"(a[5]), "=&r"(a[6]), "=&r"(a[7]), "=&r"(a[8]), "=&r"(a[9]), "=&r"(a[10]),
          "=&r"(a[11]), "=&r"(a[12]), "=&r"(a[13]), "=&r"(a[14]), "=&r"(a[15]), "=&r"(b[0]), "=&r"(b[1]), "=&r"(b[2]), "=&r"(b[3]), "=&r"(b[4]), "=&r"(b[5]),
          "=&r"(b[6]), "=&r"(b[7]), "=&r"(b[8]), "=&r"(b[9]), "=&r"(b[10]), "=&r"(b[11]), "=&r"(b[12]), "=&r"(b[13]), "=&r"(b[14]), "=&r"(b[15])
        : "r"(addr), "r"(addr + 16u)
        : "memory");
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = __uint_as_float(a[k]), v[16 + k] = __uint_as_float(b[k]);
}

// Sixteen columns of the warp's 32 rows, added over the accumulators in order (SEGMENTS: to z).
template <bool SEGMENTS = false>
__device__ __forceinline__ void lt_sums(uint32_t src, int accs, float (&z)[16])
{
    uint32_t a[16];
    if (SEGMENTS) {
        for (int i = 0; i < accs; ++i) {
            lt_read16(src + (uint32_t)(i * (kLtMaxN / accs)), a);
#pragma unroll
            for (int k = 0; k < 16; ++k) z[k] += __uint_as_float(a[k]);
        }
        return;
    }
    lt_load16(src, a);
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int k = 0; k < 16; ++k) z[k] = __uint_as_float(a[k]);
    for (int i = 1; i < accs; ++i) {
        lt_load16(src + (uint32_t)(i * (kLtMaxN / accs)), a);
        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
        for (int k = 0; k < 16; ++k) z[k] += __uint_as_float(a[k]);
    }
}

// A segment's sums of `count` columns, to their places in the slab.
__device__ __forceinline__ void lt_segment(uint32_t src, int accs, int count, float* at, bool whole, bool add)
{
    int q = 0;
    if (accs == 1) {
        for (; q + 16 < count; q += 32) {
            float z[32];
            __syncwarp();
            lt_read32(src + (uint32_t)q, z);
            lt_put(at + q * kLtM, z, whole, add);
        }
    }
    for (; q < count; q += 16) {
        float z[16];
        __syncwarp();
        lt_sums(src + (uint32_t)q, accs, z);
        lt_put(at + q * kLtM, z, whole, add);
    }
}

// Sixteen tokens (the first `count` of them) of a finished accumulator: row o of the output in each lane.  Of bf16 values, the
// lanes of a pair exchange one for every two tokens, so that each stores two rows of a token; their residual is read the same way.
template <bool SCALED>
__device__ __forceinline__ void lt_result(const LinearOut& out, uint32_t src, int accs, float b, int64_t t0, int count, int64_t o, bool live, int lane)
{
    float z[16];
    __syncwarp();
    lt_sums(src, accs, z);
    if (SCALED) {
#pragma unroll
        for (int k = 0; k < 16; ++k) z[k] = out.scaled(z[k], k < count ? __ldg(out.scale + t0 + k) : 0.0f);
    }
    const bool odd = lane & 1, both = (o | 1) < out.n, one = (o & ~(int64_t)1) < out.n;  // the pair's two rows exist, its first
    const bool paired = out.y_bf16 && out.pairs && count >= 16;
    float r[16];
    if (paired) {
        const int64_t first = (t0 + odd) * out.ld_residual + (o & ~(int64_t)1);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            uint32_t u = 0u;
            if (out.residual && one) {
                const uint16_t* p = static_cast<const uint16_t*>(out.residual) + first + 2 * k * out.ld_residual;
                u = both ? *reinterpret_cast<const uint32_t*>(p) : (uint32_t)*p;
            }
            r[2 * k] = __uint_as_float(u << 16), r[2 * k + 1] = __uint_as_float(u & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 16; ++k) r[k] = live && k < count ? out.residual_at(t0 + k, o) : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < 16; ++k) z[k] += b;
    // rows (o & ~1, + 1) of tokens 2 k + odd
    auto exchange = [&](float (&v)[16], auto&& use) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float other = __shfl_xor_sync(kFull, odd ? v[2 * k] : v[2 * k + 1], 1);
            use(k, odd ? other : v[2 * k], odd ? v[2 * k + 1] : other);
        }
    };
    auto put = [&](uint16_t* p, uint32_t u) {
        if (both) *reinterpret_cast<uint32_t*>(p) = u;
        else *p = (uint16_t)u;
    };
    if (paired) {
        const int64_t even = o & ~(int64_t)1;
        if (out.pre) {
            uint16_t* p = out.pre + (t0 + odd) * out.ld_pre + even;
            exchange(z, [&](int k, float x, float y) {
                if (one) put(p + 2 * k * out.ld_pre, bf16_pair(x, y));
            });
        }
        activate_all(z, out.act);
        uint16_t* p = static_cast<uint16_t*>(out.y) + (t0 + odd) * out.ldy + even;
        exchange(z, [&](int k, float x, float y) {
            if (one) put(p + 2 * k * out.ldy, bf16_pair(x + r[2 * k], y + r[2 * k + 1]));
        });
        return;
    }
    if (out.pre) {
#pragma unroll
        for (int k = 0; k < 16; ++k)
            if (live && k < count) out.pre[(t0 + k) * out.ld_pre + o] = bf16_round(z[k]);
    }
    activate_all(z, out.act);
    const int64_t at = t0 * out.ldy + o;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        if (!live || k >= count) continue;
        const float v = z[k] + r[k];
        if (out.y_bf16) static_cast<uint16_t*>(out.y)[at + k * out.ldy] = bf16_round(v);
        else static_cast<float*>(out.y)[at + k * out.ldy] = v;
    }
}

// N tokens of a gated tile: lane pairs have column f of the gate and of the up rows; the even lane takes the even tokens.
template <int N>
__device__ __forceinline__ void lt_pair(const LinearOut& out, float (&z)[N], float b, int64_t t0, int count, int64_t f, bool live, int lane)
{
    const bool odd = lane & 1;
#pragma unroll
    for (int k = 0; k < N; ++k) z[k] += b;
    if (out.pre && live) {
        uint16_t* const p = out.pre + t0 * out.ld_pre + (odd ? out.n : 0) + f;
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (k < count) p[k * out.ld_pre] = bf16_round(z[k]);
    }
    float g[N / 2], u[N / 2];
#pragma unroll
    for (int k = 0; k < N / 2; ++k) {
        const float other = __shfl_xor_sync(kFull, odd ? z[2 * k] : z[2 * k + 1], 1);
        g[k] = odd ? other : z[2 * k], u[k] = odd ? z[2 * k + 1] : other;
    }
    activate_gate(g, out.act);
    if (!live) return;
    const int64_t at = (t0 + odd) * out.ldy + f;
#pragma unroll
    for (int k = 0; k < N / 2; ++k) {
        if (2 * k + odd >= count) continue;
        const float v = g[k] * u[k];
        if (out.y_bf16) static_cast<uint16_t*>(out.y)[at + 2 * k * out.ldy] = bf16_round(v);
        else static_cast<float*>(out.y)[at + 2 * k * out.ldy] = v;
    }
}

template <int N>
__device__ __forceinline__ void lt_result_pair(const LinearOut& out, uint32_t src, int accs, float b, int64_t t0, int count, int64_t f, bool live, int lane)
{
    float z[N];
    __syncwarp();
#pragma unroll
    for (int q = 0; q < N; q += 16) lt_sums(src + (uint32_t)q, accs, *reinterpret_cast<float(*)[16]>(z + q));
    lt_pair(out, z, b, t0, count, f, live, lane);
}

// HALF: blocks of 32 weights, two constants per thread and k-block.  LUT: half of the codes are looked up in a table of pairs.
// GATED (forward): a tile holds 64 gate rows and the 64 up rows of the same columns of the result, in turn.
// SCALED (backward): a token's sums are multiplied by out.scale; with a test of it in every launch bof4_linear_backward took 4 % longer (200 tokens of 14336 x 4096: 44.6 us, 42.8 without).
// SEGMENTS (forward): results in fp32 of a long K, whose accumulators take at most `work.segment` lines; the segments of a part of a tile are added, rounded, in its slab.
template <bool BWD, class ST, bool HALF, bool OPQ, bool LUT, bool GATED, bool SCALED, bool SEGMENTS>
__global__ void __launch_bounds__(kLtThreads, 1)
linear_tc_kernel(const __grid_constant__ CUtensorMap code_map, const __grid_constant__ CUtensorMap token_map, const void* __restrict__ scales,
                 int64_t cols, int block_shift, int64_t last_scale, const float* __restrict__ levels, const LinearOut out,
                 int* __restrict__ status, const int* __restrict__ heads, const int2* __restrict__ nodes, const LtWork work,
                 unsigned char* __restrict__ ws, float* __restrict__ parts)
{
    extern __shared__ unsigned char s_dyn[];
    __shared__ __align__(8) unsigned long long s_full[kLtGroups], s_empty[kLtGroups], s_half_full[kLtMaxHalves],
        s_half_empty[kLtMaxHalves], s_acc_full[2], s_acc_empty[2];
    __shared__ __align__(16) float2 s_levels[8];
    __shared__ uint32_t s_tmem;
    __shared__ int s_fail, s_sums, s_sum[2];
    if (threadIdx.x == 0) tc_fetch_map(&code_map), tc_fetch_map(&token_map);
    if (!after_previous()) return;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int per_tile = work.per_tile, box_n = work.box_n;
    const uint32_t b_stage = (uint32_t)box_n * 128u;  // a multiple of 2048
    const uint32_t a_ring = (smem_u32(s_dyn) + 1023u) & ~1023u, code_ring = a_ring + (uint32_t)(kLtGroups * kLtABytes);
    const uint32_t b_ring = code_ring + (uint32_t)work.halves * kLtHalfBytes;
    const uint32_t pairs = b_ring + (uint32_t)kLtGroups * b_stage;
    const int accs = work.accs;
    // a line takes a turn of every stage: line n of this CTA the n-th
    auto time = [](int n) { return (uint32_t)n & 1u; };
    const int begin = work.start((int)blockIdx.x), finish = work.start((int)blockIdx.x + 1), lines = finish - begin;
    const int tile0 = (int)((uint32_t)begin / (uint32_t)per_tile), in0 = begin - tile0 * per_tile;
    const int segs = lines ? (in0 + lines - 1) / per_tile + 1 : 0;
    auto warp_wait = [&](unsigned long long* bar, uint32_t parity) -> bool {
        if (__all_sync(kFull, tc_wait(smem_u32(bar), parity))) return true;
        if (lane == 0) s_fail = 1;
        return false;
    };
    auto init = [&](unsigned long long* bar, int count) {
        asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory");
    };
    if (tid == 0) {
        if (blockIdx.x == 0 && !out.keep_status) *status = 0;  // long before any wait can have run out
        s_fail = s_sums = 0;
        for (int s = 0; s < kLtGroups; ++s) init(&s_full[s], 4 + 1), init(&s_empty[s], 1);  // four warps of producers, and the tokens
        for (int s = 0; s < work.halves; ++s) init(&s_half_full[s], 1), init(&s_half_empty[s], 8);
        for (int b = 0; b < 2; ++b) init(&s_acc_full[b], 1), init(&s_acc_empty[b], 4);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid >= 32 && tid < 40) s_levels[tid - 32] = make_float2(__ldg(levels + 2 * (tid - 32)), __ldg(levels + 2 * (tid - 32) + 1));
    if (warp == kLtIssue) {  // tensor memory: two accumulators of 256 columns
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(2 * kLtMaxN) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (LUT && warp < kLtIssue) fill_pairs(reinterpret_cast<float2*>(s_dyn + (pairs - smem_u32(s_dyn))), levels, tid, kLtIssue * 32);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = s_tmem;

    if (warp < kLtIssue) {
        // ---- producers
        const int group = warp >> 2, thread = (warp & 3) * 32 + lane;
        const int row = BWD ? thread & 63 : thread, half = BWD ? thread >> 6 : 0;  // of W within the k-block (backward), the tile (forward)
        // Block constants, three lines ahead (past the last line: its own again; rows of M outside the matrix: its last one): the index of the
        // thread's first weight of a line, and what a line further adds to it.
        TcConst<ST> c0, c1, c2, d0, d1, d2;
        int ct = tile0, ci = in0, unasked = lines;
        auto first_of = [&](int t, int i) -> int64_t {
            const int64_t tm = (uint32_t)t / (uint32_t)work.tiles_n, k = (int64_t)i * kLtGroups + group;
            if (GATED) return ((row & 1) * out.n + tm * (kLtM / 2) + (row >> 1)) * cols + k * kLtK;
            return BWD ? (k * kLtK + row) * cols + tm * kLtM + half * 64 : (tm * kLtM + row) * cols + k * kLtK;
        };
        int64_t weight = first_of(ct, ci);
        const int64_t line_step = BWD ? (int64_t)kLtGroups * kLtK * cols : kLtGroups * kLtK;
        auto constants = [&](TcConst<ST>& c, TcConst<ST>& d) {
            const int64_t b = weight >> block_shift;
            // (past the end of K the constants are zero, as the operand is: a product of its zeros with another row's infinity or NaN
            // would reach the sums)
            const int k = (ci * kLtGroups + group) * kLtK + (BWD ? row : 0);
            c.v = d.v = 0;
            if (k < work.k) c.load(scales, b < last_scale ? b : last_scale);
            if (HALF && k + (BWD ? 0 : 32) < work.k) d.load(scales, b + 1 < last_scale ? b + 1 : last_scale);
            if (--unasked <= 0) return;
            weight += line_step;
            if (++ci == per_tile) ci = 0, ++ct, weight = first_of(ct, 0);
        };
        if (lines) constants(c0, d0), constants(c1, d1), constants(c2, d2);
        const int* head_at = nullptr;  // OPQ: the list of the warp's part of a line's k-block, 4 * kLtGroups places further for the next line
        int in = in0, tile = tile0;
        auto head_of = [&] { return heads + (((int64_t)((uint32_t)tile / (uint32_t)work.tiles_n) * per_tile + in) * kLtGroups + group) * 4 + (warp & 3); };
        if (OPQ && lines) head_at = head_of();
        // the thread's 32 bytes of a half line: two chunks of its row (64-byte swizzle); its row of the A tile (128-byte swizzle)
        const int r = BWD ? (group & 1) * 64 + row : row, chunk = (2 * (BWD ? half : group & 1)) ^ ((r >> 1) & 3);
        const uint32_t code0 = code_ring + (uint32_t)(r * 64 + chunk * 16), code1 = code_ring + (uint32_t)(r * 64 + (chunk ^ 1) * 16);
        const uint32_t tile_at = a_ring + (uint32_t)group * kLtABytes + (uint32_t)(thread * 128 + (thread & 7) * 16);
        const uint32_t full0 = smem_u32(&s_full[group]), empty0 = smem_u32(&s_empty[group]);
        int slot = group >> 1;  // of the half line
        uint32_t par = 0;
        for (int n = 0; n < lines; ++n) {
            if (!warp_wait(&s_half_full[slot], par)) break;
            uint32_t w[8];
            const uint32_t codes = (uint32_t)slot * kLtHalfBytes;
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(code0 + codes) : "memory");
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "r"(code1 + codes) : "memory");
            const float m = c0.value(), m2 = HALF ? d0.value() : m;
            c0 = c1, c1 = c2;
            if (HALF) d0 = d1, d1 = d2;
            constants(c2, d2);
            int head = -1;
            if (OPQ) {
                head = __ldg(head_at);
                head_at += 4 * kLtGroups;
                if (++in == per_tile) {
                    in = 0, ++tile;
                    if (n + 1 < lines) head_at = head_of();
                }
            }
            // everything is decoded before the wait: what lies between a stage's release and its next use is the pipeline's slack
            uint32_t lo[4], hi[4], v[32];
            lt_table(LUT ? m2 : m, s_levels, lo, hi);
            if (LUT) {
#pragma unroll
                for (int j = 0; j < 4; ++j) tc_lookup8(w[j], make_float2(m, m), pairs, (uint32_t)lane * 8u, v + 4 * j);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) lt_lookup8(w[j], lo, hi, v + 4 * j);
                if (HALF) lt_table(m2, s_levels, lo, hi);
            }
#pragma unroll
            for (int j = 4; j < 8; ++j) lt_lookup8(w[j], lo, hi, v + 4 * j);
            if (!__all_sync(kFull, tc_wait(empty0, time(n) ^ 1u))) {
                if (lane == 0) s_fail = 1;
                break;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
                asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(tile_at ^ (uint32_t)(j << 4)), "r"(v[4 * j]), "r"(v[4 * j + 1]), "r"(v[4 * j + 2]), "r"(v[4 * j + 3]) : "memory");
            if (OPQ) {
                while (head >= 0) {  // the same list for all lanes; a lane patches its own row
                    const int2 e = __ldg(nodes + head);
                    const uint32_t place = (uint32_t)e.y >> 16;
                    if ((int)(place >> 6) == lane) {
                        const uint32_t c = place & 63u;
                        asm volatile("st.shared.u16 [%0], %1;" ::"r"((tile_at ^ ((c >> 3) << 4)) + (c & 7u) * 2u), "h"((uint16_t)e.y) : "memory");
                    }
                    head = e.x;
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            // (the codes are given back once all of them have been used: given back when only their loads had been issued, slow
            // memory let the next half line overtake them)
            if (lane == 0) {
                tc_arrive(&s_half_empty[slot]);
                asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(full0) : "memory");
            }
            if ((slot += 2) >= work.halves) slot = group >> 1, par ^= 1u;
        }
    } else if (warp == kLtIssue) {
        // ---- the issuing warp: one lane does it all (with the other lanes in step, their instructions predicated off, a
        // k-block took 500 cycles to issue)
        if (tc_elect()) {
            auto wait = [&](uint32_t bar, uint32_t parity) -> bool {
                if (tc_wait(bar, parity)) return true;
                s_fail = 1;
                return false;
            };
            const uint64_t da0 = tc_smem_desc(a_ring, BWD ? 8192u : 16u), db0 = tc_smem_desc(b_ring);
            const uint32_t full0 = smem_u32(s_full);
            // fp32 accumulator, bf16 x bf16, A M-major (backward) or K-major, B K-major, M = 128, N
            const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (BWD ? 1u << 15 : 0u) | ((uint32_t)(box_n >> 3) << 17) | ((uint32_t)(kLtM >> 4) << 24);
            constexpr uint64_t a_step = BWD ? 2048 >> 4 : 32 >> 4;  // 16 of K
            int in = in0, seg = 0, run = 0;
            uint32_t acc = 0u;
            bool ok = true;
            for (int n = 0; n < lines; ++n) {
                const uint32_t par = time(n);
                uint32_t d[kLtK / 16];  // of the instructions of a k-block
#pragma unroll
                for (int kk = 0; kk < kLtK / 16; ++kk) d[kk] = tmem + (uint32_t)((seg & 1) * kLtMaxN + (kk & (accs - 1)) * (kLtMaxN / accs));
                if (acc == 0u && !(ok = wait(smem_u32(&s_acc_empty[seg & 1]), (uint32_t)((seg >> 1) & 1) ^ 1u))) break;
                // a look at all four stages first: mostly they are full, and the looks overlap
                bool ready[kLtGroups];
#pragma unroll
                for (int j = 0; j < kLtGroups; ++j) ready[j] = tc_look(full0 + 8u * (uint32_t)j, par);
#pragma unroll
                for (int j = 0; j < kLtGroups; ++j) {
                    if (!ready[j] && !(ok = wait(full0 + 8u * (uint32_t)j, par))) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t da = da0 + (uint64_t)(j * (kLtABytes >> 4)), db = db0 + (uint64_t)(j * (b_stage >> 4));
#pragma unroll
                    for (int kk = 0; kk < kLtK / 16; ++kk) {
                        asm volatile(
                            "{\n\t.reg .pred p;\n\t"
                            "setp.ne.b32 p, %4, 0;\n\t"
                            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                            :
                            : "r"(d[kk]), "l"(da + a_step * kk), "l"(db + (uint64_t)(2 * kk)), "r"(idesc), "r"(kk < accs ? acc : 1u)
                            : "memory");
                    }
                    acc = 1u;
                    tc_commit(&s_empty[j], 1u);
                }
                if (!ok) break;
                if (++in == per_tile || n + 1 == lines) {  // the end of a part of a tile
                    tc_commit(&s_acc_full[seg & 1], 1u);
                    in = 0, ++seg, acc = 0u;
                    if (SEGMENTS) run = 0;
                } else if (SEGMENTS && ++run == work.segment) {
                    tc_commit(&s_acc_full[seg & 1], 1u);
                    ++seg, acc = 0u, run = 0;
                }
            }
        }
        __syncwarp();
    } else if (warp == kLtTokens) {
        // ---- the B operand: 64 of K of the tile's tokens
        if (tc_elect()) {
            int tile = tile0, in = in0;
            bool ok = true;
            for (int n = 0; ok && n < lines; ++n) {
                const int t0 = (int)((uint32_t)tile % (uint32_t)work.tiles_n) * box_n;
                for (int j = 0; j < kLtGroups; ++j) {
                    if (!(ok = tc_wait(smem_u32(&s_empty[j]), time(n) ^ 1u))) break;
                    tc_load_box(b_ring + (uint32_t)j * b_stage, &token_map, &s_full[j], b_stage, (in * kLtGroups + j) * kLtK, t0);
                }
                if (++in == per_tile) in = 0, ++tile;
            }
            if (!ok) s_fail = 1;
        }
        __syncwarp();
    } else if (warp == kLtCodes) {
        // ---- codes: half h of line `in` of a tile, brought into L2 kLtAhead lines before
        if (tc_elect()) {
            int tile = tile0, in = in0, slot = 0, pt = tile0, pi = in0;
            uint32_t par = 0;
            bool ok = true;
            auto x_of = [&](int t, int i, int h) { return BWD ? (int)((uint32_t)t / (uint32_t)work.tiles_n) * 64 : i * 128 + h * 64; };
            auto y_of = [&](int t, int i, int h) { return BWD ? i * 256 + h * 128 : (int)((uint32_t)t / (uint32_t)work.tiles_n) * kLtM; };
            for (int n = 0; n < kLtAhead; ++n)
                if (++pi == per_tile) pi = 0, ++pt;
            for (int n = 0; ok && n < lines; ++n) {
                if (n + kLtAhead < lines) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (GATED)
                            asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global [%0, {%1, 0, %2}];" ::"l"(reinterpret_cast<uint64_t>(&code_map)),
                                         "r"(x_of(pt, pi, h)), "r"(y_of(pt, pi, h) >> 1)
                                         : "memory");
                        else asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global [%0, {%1, %2}];" ::"l"(reinterpret_cast<uint64_t>(&code_map)),
                                     "r"(x_of(pt, pi, h)), "r"(y_of(pt, pi, h))
                                     : "memory");
                    }
                    if (++pi == per_tile) pi = 0, ++pt;
                }
                for (int h = 0; h < 2; ++h) {
                    if (!(ok = tc_wait(smem_u32(&s_half_empty[slot]), par ^ 1u))) break;
                    if (GATED) tc_load_box3(code_ring + (uint32_t)slot * kLtHalfBytes, &code_map, &s_half_full[slot], kLtHalfBytes, x_of(tile, in, h), 0, y_of(tile, in, h) >> 1);
                    else tc_load_box(code_ring + (uint32_t)slot * kLtHalfBytes, &code_map, &s_half_full[slot], kLtHalfBytes, x_of(tile, in, h), y_of(tile, in, h));
                    if (++slot == work.halves) slot = 0, par ^= 1u;
                }
                if (++in == per_tile) in = 0, ++tile;
            }
            if (!ok) s_fail = 1;
        }
        __syncwarp();
    } else if (warp >= kLtResults) {
        // ---- results of the parts of tiles
        const int f = tid - kLtResults * 32, m = (warp & 3) * 32 + lane;
        unsigned long long* const tickets = reinterpret_cast<unsigned long long*>(ws);
        if (f == 0 && segs) {
            if (in0 || lines < per_tile) tc_ticket_open(tickets + tile0, work.epoch);
            if (segs > 1 && (in0 + lines) % per_tile) tc_ticket_open(tickets + tile0 + segs - 1, work.epoch);
        }
        auto sync = [] { asm volatile("bar.sync 1, 128;" ::: "memory"); };
        auto all4 = [](bool ok) -> bool {
            uint32_t r;
            asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"(ok ? 1u : 0u) : "memory");
            return r != 0u;
        };
        int done = 0;  // accumulators that were read, but for the last one of each part
        const int slab_at = (lane >> 3) * kLtM + (warp & 3) * 32 + (lane & 7) * 4;
        for (int seg = 0; seg < segs; ++seg) {
            const int tile = tile0 + seg, t0 = tile * per_tile;
            bool summed = false;
            if (SEGMENTS) {  // the segments of this part of the tile but for the last
                const int from = begin > t0 ? begin : t0, to = finish < t0 + per_tile ? finish : t0 + per_tile;
                const bool whole = to - from == per_tile;
                const int64_t first = (int64_t)((uint32_t)tile % (uint32_t)work.tiles_n) * box_n;
                const int count = (int)(out.tokens - first < box_n ? out.tokens - first : box_n);
                float* const at = parts + (2 * (int64_t)blockIdx.x + (begin <= t0 ? 1 : 0)) * kLtM * box_n + (whole ? slab_at : m);
                bool ok = true;
                for (int left = (to - from - 1) / work.segment; left; --left, ++done) {
                    const int buf = (seg + done) & 1;
                    if (!(ok = all4(warp_wait(&s_acc_full[buf], (uint32_t)((seg + done) >> 1) & 1u)))) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    lt_segment(tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(buf * kLtMaxN), accs, count, at, whole, summed);
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) tc_arrive(&s_acc_empty[buf]);
                    summed = true;
                }
                if (!ok) break;
            }
            const int buf = (seg + done) & 1;
            if (!all4(warp_wait(&s_acc_full[buf], (uint32_t)((seg + done) >> 1) & 1u))) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const int64_t o = (int64_t)((uint32_t)tile / (uint32_t)work.tiles_n) * kLtM + m, token0 = (int64_t)((uint32_t)tile % (uint32_t)work.tiles_n) * box_n;
            const int count = (int)(out.tokens - token0 < box_n ? out.tokens - token0 : box_n);
            const bool all = begin <= t0 && finish >= t0 + per_tile, live = (GATED ? o >> 1 : o) < out.n;
            const uint32_t src = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(buf * kLtMaxN);
            float* const part = parts + (2 * (int64_t)blockIdx.x + (begin <= t0 ? 1 : 0)) * kLtM * box_n;
            if (SEGMENTS && summed) {
                if (!all) {
                    lt_segment(src, accs, count, part + m, false, true);
                } else {
                    const float b = GATED && live ? out.bias_at((o & 1) * out.n + (o >> 1)) : 0.0f;
                    float* const y = static_cast<float*>(out.y) + token0 * out.ldy + o;
                    for (int q = 0; q < count; q += 32) {
                        float z[32];
                        lt_before(part + slab_at, q, count, z);
                        __syncwarp();
#pragma unroll
                        for (int h = 0; h < 32; h += 16)
                            if (q + h < count) lt_sums<true>(src + (uint32_t)(q + h), accs, *reinterpret_cast<float(*)[16]>(z + h));
                        if (GATED) {
                            lt_pair(out, z, b, token0 + q, count - q, o >> 1, live, lane);
                        } else {  // logits: nothing but stores
#pragma unroll
                            for (int k = 0; k < 32; ++k)
                                if (live && q + k < count) y[(q + k) * out.ldy] = z[k];
                        }
                    }
                }
            } else if (!all) {
                float* to = part + m;
                for (int q = 0; q < count; q += 16, to += 16 * kLtM) {
                    float z[16];
                    lt_sums(src + (uint32_t)q, accs, z);
#pragma unroll
                    for (int k = 0; k < 16; ++k) to[k * kLtM] = z[k];  // (count is padded to 16 in the workspace)
                }
            } else {
                const float b = live ? out.bias_at(GATED ? (o & 1) * out.n + (o >> 1) : o) : 0.0f;
                if (GATED) {
                    int q = 0;
                    for (; q + 16 < count; q += 32) lt_result_pair<32>(out, src + (uint32_t)q, accs, b, token0 + q, count - q, o >> 1, live, lane);
                    if (q < count) lt_result_pair<16>(out, src + (uint32_t)q, accs, b, token0 + q, count - q, o >> 1, live, lane);
                } else for (int q = 0; q < count; q += 16) lt_result<SCALED>(out, src + (uint32_t)q, accs, b, token0 + q, count - q, o, live, lane);
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) tc_arrive(&s_acc_empty[buf]);
            if (all) continue;
            const int others = work.owner(t0 + per_tile - 1) - work.owner(t0);
            __threadfence();
            sync();
            if (f == 0 && (int)(atomicAdd(tickets + tile, 1ull) & 255ull) == others) {
                tickets[tile] = 0ull;
                s_sum[s_sums++] = tile;
            }
        }
    }
    // Every loop above is bounded, so every warp gets here.
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (s_fail) {
        if (tid == 0) atomicExch(status, 1);
        tc_settle();
    }
    for (int k = 0; k < s_sums; ++k) {  // the parts in the order of the CTAs; all but the first begin inside the tile
        const int tile = s_sum[k], t0 = tile * per_tile, i0 = work.owner(t0), more = work.owner(t0 + per_tile - 1) - i0;
        const int64_t o0 = (int64_t)((uint32_t)tile / (uint32_t)work.tiles_n) * kLtM, token0 = (int64_t)((uint32_t)tile % (uint32_t)work.tiles_n) * box_n;
        const int count = (int)(out.tokens - token0 < box_n ? out.tokens - token0 : box_n);
        const int64_t slab = (int64_t)(kLtM / 4) * box_n;
        __threadfence();
        const float4* head = reinterpret_cast<const float4*>(parts) + (int64_t)(2 * i0 + (work.start(i0) <= t0 ? 1 : 0)) * slab;
        const float4* next = reinterpret_cast<const float4*>(parts) + (int64_t)(2 * i0 + 2) * slab;
        constexpr int B = 4;  // quads of rows of a thread at a time
        for (int e0 = tid; e0 < count * (kLtM / 4); e0 += B * kLtThreads) {
            float4 sum[B];
#pragma unroll
            for (int u = 0; u < B; ++u) {
                const int e = e0 + u * kLtThreads;
                sum[u] = e < count * (kLtM / 4) ? __ldcg(head + e) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            for (int i = 0; i < more; i += 2) {
                float4 v[2][B];
#pragma unroll
                for (int w = 0; w < 2; ++w)
#pragma unroll
                    for (int u = 0; u < B; ++u) {
                        const int e = e0 + u * kLtThreads;
                        v[w][u] = i + w < more && e < count * (kLtM / 4) ? __ldcg(next + (int64_t)(2 * (i + w)) * slab + e) : make_float4(0.f, 0.f, 0.f, 0.f);
                    }
#pragma unroll
                for (int w = 0; w < 2; ++w)
#pragma unroll
                    for (int u = 0; u < B; ++u) sum[u].x += v[w][u].x, sum[u].y += v[w][u].y, sum[u].z += v[w][u].z, sum[u].w += v[w][u].w;
            }
            if constexpr (GATED) {
#pragma unroll
                for (int u = 0; u < B; ++u) {
                    const int e = e0 + u * kLtThreads;
                    if (e < count * (kLtM / 4)) out.store_pairs(sum[u], token0 + (e >> 5), (o0 >> 1) + (e & 31) * 2);
                }
            } else {
                LinearFour four[B];
#pragma unroll
                for (int u = 0; u < B; ++u) {
                    const int e = e0 + u * kLtThreads;
                    if (e < count * (kLtM / 4) && o0 + (e & 31) * 4 < out.n) four[u].residual(out, token0 + (e >> 5), o0 + (e & 31) * 4);
                }
#pragma unroll
                for (int u = 0; u < B; ++u) {
                    const int e = e0 + u * kLtThreads;
                    const int64_t o = o0 + (e & 31) * 4;
                    if (SCALED && e < count * (kLtM / 4)) {
                        const float f = __ldg(out.scale + token0 + (e >> 5));
                        sum[u] = make_float4(out.scaled(sum[u].x, f), out.scaled(sum[u].y, f), out.scaled(sum[u].z, f), out.scaled(sum[u].w, f));
                    }
                    if (e < count * (kLtM / 4) && o < out.n) four[u].store(out, sum[u], token0 + (e >> 5), o);
                }
            }
        }
    }
    if (warp == kLtIssue)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * kLtMaxN) : "memory");
}

// A launch, and the kernel's variant for it.  The forward, backward, scaled and gated variants are compiled in files of their own.
struct LtLaunch {
    const CUtensorMap *code_map, *token_map;
    const LinearW* w;
    const LinearOut* out;
    int* status;
    const int* heads;  // NULL without a list
    const int2* nodes;
    const LtWork* work;
    int ctas;
    unsigned char* ws;
    float* parts;
    cudaStream_t st;
};
int linear_tc_forward(const LtLaunch& go);
int linear_tc_backward(const LtLaunch& go);
int linear_tc_scaled(const LtLaunch& go);
int linear_tc_gated(const LtLaunch& go);
int linear_tc_forward_segments(const LtLaunch& go);
int linear_tc_gated_segments(const LtLaunch& go);

template <bool BWD, class ST, bool HALF, bool OPQ, bool LUT, bool GATED, bool SCALED, bool SEGMENTS>
int lt_go(const LtLaunch& go)
{
    constexpr auto kern = linear_tc_kernel<BWD, ST, HALF, OPQ, LUT, GATED, SCALED, SEGMENTS>;
    if (const int rc = ensure_dynamic_smem<kern>(kLtSmem)) return rc;
    const LinearW& w = *go.w;
    launch_after(kern, go.ctas, kLtThreads, kLtSmem, go.st, *go.code_map, *go.token_map, w.scales, w.cols, w.block_shift, w.rows * w.cols / w.block_size - 1,
                 w.levels, *go.out, go.status, go.heads, go.nodes, *go.work, go.ws, go.parts);
    return BOF4_OK;
}
template <bool BWD, bool GATED, bool SCALED, bool SEGMENTS, class ST, bool HALF>
int lt_pick(const LtLaunch& go)
{
    if (go.heads) return go.work->table ? lt_go<BWD, ST, HALF, true, true, GATED, SCALED, SEGMENTS>(go) : lt_go<BWD, ST, HALF, true, false, GATED, SCALED, SEGMENTS>(go);
    return go.work->table ? lt_go<BWD, ST, HALF, false, true, GATED, SCALED, SEGMENTS>(go) : lt_go<BWD, ST, HALF, false, false, GATED, SCALED, SEGMENTS>(go);
}
template <bool BWD, bool GATED, bool SCALED = false, bool SEGMENTS = false>
int lt_launch(const LtLaunch& go)
{
    const bool half = go.w->block_size == 32;
    if (go.w->scale_dtype == BOF4_F32) return half ? lt_pick<BWD, GATED, SCALED, SEGMENTS, F32, true>(go) : lt_pick<BWD, GATED, SCALED, SEGMENTS, F32, false>(go);
    return half ? lt_pick<BWD, GATED, SCALED, SEGMENTS, BF16, true>(go) : lt_pick<BWD, GATED, SCALED, SEGMENTS, BF16, false>(go);
}

}  // namespace bof4
