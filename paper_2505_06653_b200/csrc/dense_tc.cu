// Products of many tokens with a decoded matrix on the tensor cores:  z[t, o] = sum_k a[t, k] b[o, k]  (or b[k, o]).
//
// From some hundred tokens on a weight is used so often that it is decoded once, by bof4_dequantize, and both operands are
// plain bf16.  Two SMs (a cluster) share a tile of 256 tokens by 256 columns: tcgen05.mma with cta_group::2 and M = 256, each SM
// holding the rows of 128 tokens and half of the columns' rows.  So a k-block of 64 takes 32 KiB of each SM's shared memory
// in and out, 512 of the 128-byte cycles of its data path, as long as the products themselves take (a tile of 128 x 256
// of one SM takes 768: linear_tc.cuh).
//
//   1 loads    TMA loads of both operands, six or seven stages; those of both SMs complete the first SM's barrier
//   1 issuer   in the first SM: four instructions (K = 16) per k-block
//   16 results a warp has 32 tokens and a quarter of the columns of a finished accumulator (there are two); a lane keeps the 64
//              sums of its token in registers
//
// The tensor cores cut a sum off at every step of 16 of K, so an accumulator takes a segment of K only, and the segments are added in
// registers, rounded.  Results in fp32 (and logits) have segments of 1024 of K: losses with K = 4096 are off by 0.6e-6 in 2-norms, by 1.4e-6 with segments of
// 2048, 3.6e-6 with one accumulator.  That is nothing beside a rounding to bf16 (1.7e-3), and results that wait for an accumulator to be read hold the next
// one up, so results in bf16 have longer ones (4096 tokens by 128256 x 4096 with the gradient: 1 % between segments of 1024 and 2048).
//
// What bounds it: with all SMs at work the power limit, 1.55 to 1.63 PFLOP/s in a cold launch (28672 x 4096 by 4096 tokens 622 us, tensor cores busy 81 to 86 % of the time at
// 1024 tokens), 1.2 to 1.3 in a row of calls; with 48 of the 74 pairs at work a k-block takes the 512 cycles that it has to.  A lane has a token's results, so that each store
// of a warp goes to 32 rows: whole sectors of 32 bytes instead of halves took a gated block of 4096 tokens from 847 to 760 us, a loss with its gradient from 7.3 to 7.0 ms.
// 18 warps have 96 registers a thread: the products that store or add spill 16 and 24 bytes, the logits 36, the gated ones 236 and (rows at odd places) 324 where they finish a tile.
//
// Tiles go to the clusters in turn.  What is left after the last whole round is cut along K into as many parts as there are clusters for
// (74 / tiles, at most eight) where K is long enough to pay for it.  They come first; the sums of a
// tile's parts are added in order by the SM that completes it last (a ticket: nobody waits).  256 tiles on 74 clusters take 3.5 rounds that way.  Equal shares of all k-blocks for every cluster (3.46 rounds) lost more
// than that: clusters that stand at different places of K find nothing of one another's in L2 (4096 x 4096, K = 16384: 412 us).
//
// Every wait is bounded: a time-out sets the status word, everybody leaves, the kernel frees its tensor memory and returns.
#include "dense_tc.cuh"

namespace bof4 {

constexpr int kDnM = 256, kDnN = 256, kDnK = 64;
template <int USE>
constexpr int dn_stages = USE == kDenseGatedRows ? 6 : 7;  // (results that go through shared memory need room of their own)
constexpr int kDnHalf = 128 * kDnK * 2;         // an SM's part of an operand in a stage
constexpr int kDnStage = 2 * kDnHalf;
constexpr int kDnSmem = 7 * kDnStage + 1024;
constexpr int kDnBlock = 32 * 8 * 4;            // a warp's block of results on their way out: 32 rows of 8 words
constexpr int kDnResults = 16, kDnCols = 64;    // warps that read results, columns of each
constexpr int kDnLoads = kDnResults, kDnIssue = kDnResults + 1;
constexpr int kDnThreads = 32 * (kDnResults + 2);
constexpr int kDnClusters = kSMs / 2;
constexpr int kDnMaxParts = 8;                  // of a tile
constexpr int kDnGroup = 16;                    // tiles of tokens that are gone through before the next columns: with K = 4096, 32 MiB of L2

__device__ __forceinline__ uint32_t dn_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t dn_first_sm(uint32_t addr)  // the same place in the cluster's first SM
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}
__device__ __forceinline__ void dn_cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void dn_load2(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 :
                 : "r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y)
                 : "memory");
}
__device__ __forceinline__ void dn_load3(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z)
{
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 :
                 : "r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y), "r"(z)
                 : "memory");
}
__device__ __forceinline__ void dn_commit(uint32_t bar)  // on the barriers of both SMs
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void dn_read16(uint32_t addr, uint32_t (&v)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
          "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(addr)
        : "memory");
}

// The units of work of a cluster in order: k-blocks k0 ... k1 - 1 of a tile.
struct DenseWalk {
    int next;
    int unit, tile, k0, k1;
    __device__ __forceinline__ explicit DenseWalk(int cluster) : next(cluster) {}
    __device__ __forceinline__ bool step(const DenseWork& w)
    {
        unit = next;
        const int cut = w.split * w.parts;
        if (unit < cut) {
            tile = unit / w.parts;
            const int part = unit - tile * w.parts;
            k0 = w.per_tile * part / w.parts, k1 = w.per_tile * (part + 1) / w.parts;
        } else {
            tile = unit - cut + w.split;
            if (tile >= w.tiles_m * w.tiles_n) return false;
            k0 = 0, k1 = w.per_tile;
        }
        next += w.clusters;
        return true;
    }
};
__device__ __forceinline__ void dn_place(const DenseWork& w, int tile, int& m, int& n)
{
    const int per_group = kDnGroup * w.tiles_n, g = (int)((uint32_t)tile / (uint32_t)per_group), in = tile - g * per_group;
    const int left = w.tiles_m - g * kDnGroup, width = left < kDnGroup ? left : kDnGroup;
    n = (int)((uint32_t)in / (uint32_t)width);
    m = g * kDnGroup + in - n * width;
}

// A lane's results lie in its token's row, 32 bytes of it at a time where they can: whole sectors, half of the instructions.
__device__ __forceinline__ void dn_put32(void* p, const uint32_t (&v)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]),
                 "r"(v[7])
                 : "memory");
}
__device__ __forceinline__ void dn_get32(const void* p, uint32_t (&v)[8])
{
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "l"(p)
                 : "memory");
}
// Sixteen neighbouring values, `count` of them in the row, which begins at a multiple of `align` bytes.  (Rows of odd length begin at odd places in turn.)
__device__ __forceinline__ void dn_store16(uint16_t* p, const float* v, int count, int align)
{
    if (count < 16) {
#pragma unroll
        for (int k = 0; k < 16; ++k)
            if (k < count) p[k] = bf16_round(v[k]);
        return;
    }
    if (align < 4 && (reinterpret_cast<uintptr_t>(p) & 2u)) {
        p[0] = bf16_round(v[0]), p[15] = bf16_round(v[15]);
#pragma unroll
        for (int k = 1; k < 15; k += 2) *reinterpret_cast<uint32_t*>(p + k) = bf16_pair(v[k], v[k + 1]);
        return;
    }
    uint32_t w[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = bf16_pair(v[2 * k], v[2 * k + 1]);
    if (align >= 32) {
        dn_put32(p, w);
    } else if (align >= 16) {
        reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]), reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    } else if (align >= 8) {
#pragma unroll
        for (int k = 0; k < 4; ++k) reinterpret_cast<uint2*>(p)[k] = make_uint2(w[2 * k], w[2 * k + 1]);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) reinterpret_cast<uint32_t*>(p)[k] = w[k];
    }
}
__device__ __forceinline__ void dn_store16(float* p, const float* v, int count)  // rows at multiples of 32 bytes
{
    if (count < 16) {
#pragma unroll
        for (int k = 0; k < 16; ++k)
            if (k < count) p[k] = v[k];
        return;
    }
#pragma unroll
    for (int h = 0; h < 16; h += 8) {
        uint32_t w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = __float_as_uint(v[h + k]);
        dn_put32(p + h, w);
    }
}

// Eight words of each lane's row, through shared memory: a store of the warp goes to four rows, wherever they begin.  p: the lane's row, `count` elements
// of bf16 (two a word) or fp32 of it exist; rows of bf16 may begin at odd elements.  All lanes take part.
template <class T>
__device__ __forceinline__ void dn_rows(uint32_t block, const uint32_t (&w)[8], T* p, bool live, int count, int lane)
{
    constexpr int E = sizeof(T) == 2 ? 2 : 1;
    __syncwarp();
#pragma unroll
    for (uint32_t c = 0; c < 2; ++c)  // without meeting a bank twice
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(block + (uint32_t)(lane * 32) + ((c ^ (uint32_t)(lane >> 2 & 1)) << 4)), "r"(w[4 * c]), "r"(w[4 * c + 1]),
                     "r"(w[4 * c + 2]), "r"(w[4 * c + 3])
                     : "memory");
    __syncwarp();
    const int l = lane & 7;
    const unsigned int rows = __ballot_sync(kFull, live);
#pragma unroll 4
    for (int i = 0; i < 8; ++i) {
        const int r = 4 * i + (lane >> 3);
        uint32_t v;
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(block + (uint32_t)(r * 32) + (((uint32_t)(l >> 2) ^ (uint32_t)(r >> 2 & 1)) << 4) + (uint32_t)(l & 3) * 4u) : "memory");
        T* const q = reinterpret_cast<T*>(__shfl_sync(kFull, reinterpret_cast<unsigned long long>(p), r)) + E * l;
        if (!(rows >> r & 1u) || E * l >= count) continue;
        if (E == 1 || (E * l + 1 < count && !(reinterpret_cast<uintptr_t>(q) & 2u))) {
            *reinterpret_cast<uint32_t*>(q) = v;
        } else {
            uint16_t* const h = reinterpret_cast<uint16_t*>(q);
            h[0] = (uint16_t)v;
            if (E * l + 1 < count) h[1] = (uint16_t)(v >> 16);
        }
    }
}
// Sixteen values of each lane's row: from the lanes where rows begin at multiples of 32 bytes, through shared memory elsewhere (1022 tokens by 1088 columns, z kept:
// 13376 columns of the result 67 us from the lanes and 77 through shared memory, 13384 95 and 76, 13382 206 and 84).
template <bool ROWS>
__device__ __forceinline__ void dn_put16(uint32_t block, uint16_t* p, const float* v, bool live, int count, int align, int lane)
{
    if constexpr (ROWS) {
        if (align < 32) {
            uint32_t w[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) w[k] = bf16_pair(v[2 * k], v[2 * k + 1]);
            dn_rows(block, w, p, live, count, lane);
            return;
        }
    }
    if (live) dn_store16(p, v, count, 32);
}
template <bool ROWS>
__device__ __forceinline__ void dn_put16(uint32_t block, float* p, const float* v, bool live, int count, int align, int lane)
{
    if constexpr (ROWS) {
        if (align < 32) {
#pragma unroll
            for (int h = 0; h < 16; h += 8) {
                uint32_t w[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) w[k] = __float_as_uint(v[h + k]);
                dn_rows(block, w, p + h, live, count - h, lane);
            }
            return;
        }
    }
    if (live) dn_store16(p, v, count);
}

// What is known of a token before its sums are.
struct DenseToken {
    int64_t target;
    float ref;  // add: the factor
};
template <int USE>
__device__ __forceinline__ DenseToken dn_token(const DenseOut& out, int64_t t)
{
    DenseToken k{-1, 0.0f};
    if (t >= out.tokens) return k;
    if (USE == kDenseLoss) {
        k.target = __ldg(out.targets + t);
        if (!out.first) k.ref = __ldg(out.ref + t);
    }
    if (USE == kDenseAdd && out.factor) k.ref = __ldg(out.factor + t);
    return k;
}

// A token's sums of columns o0 ... o0 + 63 of z, gate and up in turn: columns o0 / 2 ... of y.  (All lanes of the warp take part.)  ROWS: some rows begin at odd places;
// with the code and the room for them in every launch, 4096 tokens of 28672 x 4096 took 776 us, 745 without.
template <bool ROWS>
__device__ __forceinline__ void dn_gated(const DenseOut& out, float (&z)[kDnCols], int64_t t, int64_t o0, uint32_t block, int lane)
{
    const int64_t f0 = o0 >> 1;
    const int left = (int)(out.n - f0 < 32 ? out.n - f0 : 32);
    const bool live = t < out.tokens;
    if (left <= 0) return;
    if (out.bias) {
#pragma unroll
        for (int j = 0; j < kDnCols / 2; ++j) {
            if (j < left) {
                const int64_t f = f0 + j;
                z[2 * j] += out.bias_bf16 ? bf16_value(__ldg(static_cast<const uint16_t*>(out.bias) + f)) : __ldg(static_cast<const float*>(out.bias) + f);
                z[2 * j + 1] += out.bias_bf16 ? bf16_value(__ldg(static_cast<const uint16_t*>(out.bias) + out.n + f))
                                              : __ldg(static_cast<const float*>(out.bias) + out.n + f);
            }
        }
    }
#pragma unroll
    for (int c = 0; c < kDnCols / 32; ++c) {
        const int count = left - 16 * c;
        if (count <= 0) break;
        float g[16], u[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) g[k] = z[32 * c + 2 * k], u[k] = z[32 * c + 2 * k + 1];
        if (out.pre) {
            uint16_t* const p = out.pre + t * out.ld_pre + f0 + 16 * c;
            dn_put16<ROWS>(block, p, g, live, count, out.pre_align, lane);
            dn_put16<ROWS>(block, p + out.n, u, live, count, out.pre_align, lane);
        }
        activate_gate(g, out.act);
#pragma unroll
        for (int k = 0; k < 16; ++k) g[k] *= u[k];
        const int64_t at = t * out.ldy + f0 + 16 * c;
        if (out.y_bf16) dn_put16<ROWS>(block, static_cast<uint16_t*>(out.y) + at, g, live, count, out.align, lane);
        else dn_put16<ROWS>(block, static_cast<float*>(out.y) + at, g, live, count, out.align, lane);
    }
}

// The same of the other products.
template <int USE>
__device__ __forceinline__ void dn_finish(const DenseOut& out, const DenseToken& token, float (&z)[kDnCols], int64_t t, int64_t o0)
{
    if (t >= out.tokens) return;
    const int left = (int)(out.n - o0 < kDnCols ? out.n - o0 : kDnCols);
    if (left <= 0) return;
    if (USE == kDenseStore) {
        uint16_t* const p = static_cast<uint16_t*>(out.y) + t * out.ldy + o0;
#pragma unroll
        for (int c = 0; c < kDnCols / 16; ++c)
            if (16 * c < left) dn_store16(p + 16 * c, z + 16 * c, left - 16 * c, out.align);
    }
    if (USE == kDenseAdd) {  // (rows of y hold multiples of 32 values)
        float* const p = static_cast<float*>(out.y) + t * out.ldy + o0;
#pragma unroll
        for (int c = 0; c < kDnCols / 8; ++c) {
            if (8 * c >= left) break;
            uint32_t v[8];
            if (out.factor) {
                dn_get32(p + 8 * c, v);
#pragma unroll
                for (int k = 0; k < 8; ++k) z[8 * c + k] = fmaf(__uint_as_float(v[k]), token.ref, z[8 * c + k]);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = __float_as_uint(z[8 * c + k]);
            dn_put32(p + 8 * c, v);
        }
    }
    if (USE == kDenseLoss) {
        // Exponentials against the token's reference, or this part's own maximum where it lies far above (or, where the reference is only a
        // guess, far below): any reference within a factor e^24 leaves sums and products far inside the range of fp32 and bf16.
        // The target's logit is kept, and has no part in the sums.
        const int64_t target = token.target - out.first_row - o0;
        const bool inside = target >= 0 && target < left;
        const int at = inside ? (int)target : -1;
        float top = -INFINITY, own = 0.0f;
#pragma unroll
        for (int k = 0; k < kDnCols; ++k) {
            own = k == at ? z[k] : own;
            z[k] = k == at || k >= left ? -INFINITY : z[k];
            top = fmaxf(top, z[k]);
        }
        if (inside) out.target_logit[t] = own;
        float ref = token.ref;
        if (top > ref + 24.0f || (out.first && top < ref - 24.0f && top > -INFINITY)) ref = top;
        if (ref == -INFINITY) ref = 0.0f;  // nothing but infinitely unlikely rows so far
        float sum = 0.0f;
        uint16_t* const p = static_cast<uint16_t*>(out.y) + t * out.ldy + o0;
#pragma unroll
        for (int c = 0; c < kDnCols / 16; ++c) {
            float s = 0.0f;
            uint32_t e[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float a = __expf(z[16 * c + 2 * k] - ref), b = __expf(z[16 * c + 2 * k + 1] - ref);
                s += a, s += b;
                e[k] = bf16_pair(a, b);
            }
            sum += s;
            if (out.y && 16 * c < left) dn_put32(p + 16 * c, e);  // (rows are padded to 256)
        }
        out.stats[(o0 / kDnCols) * out.tokens + t] = make_float2(ref, sum);
    }
}

template <int USE, bool NMAJOR>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kDnThreads, 1)
dense_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map, const DenseOut out, int* __restrict__ status,
             const DenseWork work, unsigned long long* __restrict__ tickets, float* __restrict__ parts)
{
    constexpr int kDnStages = dn_stages<USE>;
    constexpr bool kGated = USE == kDenseGated || USE == kDenseGatedRows;
    extern __shared__ unsigned char s_dyn[];
    __shared__ __align__(8) unsigned long long s_full[kDnStages], s_empty[kDnStages], s_acc_full[2], s_acc_empty[2];
    __shared__ uint32_t s_tmem;
    __shared__ int s_fail, s_last;
    if (threadIdx.x == 0) tc_fetch_map(&a_map), tc_fetch_map(&b_map);
    if (!after_previous()) return;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = (int)dn_rank(), cluster = (int)blockIdx.x >> 1;
    const uint32_t ring = (smem_u32(s_dyn) + 1023u) & ~1023u;
    auto init = [&](unsigned long long* bar, int count) {
        asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory");
    };
    if (tid == 0) {
        if (blockIdx.x == 0 && !out.keep_status) *status = 0;  // long before any wait can have run out
        s_fail = 0;
        for (int s = 0; s < kDnStages; ++s) init(&s_full[s], 1), init(&s_empty[s], 1);
        for (int b = 0; b < 2; ++b) init(&s_acc_full[b], 1), init(&s_acc_empty[b], 2 * kDnResults);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kDnIssue) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(2 * kDnN) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    dn_cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = s_tmem;
    DenseWalk walk(cluster);

    if (warp == kDnLoads) {
        if (tc_elect()) {
            int stage = 0;
            uint32_t turn = 0;
            bool ok = true;
            while (ok && walk.step(work)) {
                int m, n;
                dn_place(work, walk.tile, m, n);
                const int t0 = m * kDnM + rank * 128, o0 = n * kDnN + rank * 128;
                for (int k = walk.k0; k < walk.k1; ++k) {
                    if (!(ok = tc_wait(smem_u32(&s_empty[stage]), turn ^ 1u))) break;
                    if (rank == 0)  // what both SMs load
                        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(&s_full[stage])), "r"(2 * kDnStage) : "memory");
                    const uint32_t bar = dn_first_sm(smem_u32(&s_full[stage])), at = ring + (uint32_t)stage * kDnStage;
                    dn_load2(at, &a_map, bar, k * kDnK, t0);
                    if (kGated) {
                        dn_load3(at + kDnHalf, &b_map, bar, k * kDnK, 0, o0 >> 1);
                    } else if (NMAJOR) {
                        dn_load2(at + kDnHalf, &b_map, bar, o0, k * kDnK);
                        dn_load2(at + kDnHalf + kDnHalf / 2, &b_map, bar, o0 + 64, k * kDnK);
                    } else {
                        dn_load2(at + kDnHalf, &b_map, bar, k * kDnK, o0);
                    }
                    if (++stage == kDnStages) stage = 0, turn ^= 1u;
                }
            }
            if (!ok) s_fail = 1;
        }
        __syncwarp();
    } else if (warp == kDnIssue) {
        if (rank == 0 && tc_elect()) {
            const uint64_t a0 = tc_smem_desc(ring), b0 = tc_smem_desc(ring + kDnHalf, NMAJOR ? 8192u : 16u);
            // fp32 accumulator, bf16 x bf16, A K-major, B N-major or K-major, N = 256, M = 256
            const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (NMAJOR ? 1u << 16 : 0u) | ((uint32_t)(kDnN >> 3) << 17) | ((uint32_t)(kDnM >> 4) << 24);
            constexpr uint64_t b_step = NMAJOR ? 2048 >> 4 : 32 >> 4;  // 16 of K
            int stage = 0, seg = 0;
            uint32_t turn = 0;
            bool ok = true;
            while (ok && walk.step(work)) {
                for (int k = walk.k0; ok && k < walk.k1; ++seg) {
                    if (!(ok = tc_wait(smem_u32(&s_acc_empty[seg & 1]), (uint32_t)((seg >> 1) & 1) ^ 1u))) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t d = tmem + (uint32_t)((seg & 1) * kDnN);
                    const int end = walk.k1 < k + work.segment ? walk.k1 : k + work.segment;
                    for (uint32_t acc = 0u; k < end; ++k, acc = 1u) {
                        if (!(ok = tc_wait(smem_u32(&s_full[stage]), turn))) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint64_t da = a0 + (uint64_t)(stage * (kDnStage >> 4)), db = b0 + (uint64_t)(stage * (kDnStage >> 4));
#pragma unroll
                        for (int kk = 0; kk < kDnK / 16; ++kk)
                            asm volatile(
                                "{\n\t.reg .pred p;\n\t"
                                "setp.ne.b32 p, %4, 0;\n\t"
                                "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                                :
                                : "r"(d), "l"(da + (uint64_t)(2 * kk)), "l"(db + b_step * kk), "r"(idesc), "r"(kk ? 1u : acc)
                                : "memory");
                        dn_commit(smem_u32(&s_empty[stage]));
                        if (++stage == kDnStages) stage = 0, turn ^= 1u;
                    }
                    if (ok) dn_commit(smem_u32(&s_acc_full[seg & 1]));
                }
            }
            if (!ok) s_fail = 1;
        }
        __syncwarp();
    } else {
        // ---- results: tokens 32 * quarter + lane of this SM's 128, a quarter of the columns
        const int quarter = warp & 3, part = warp >> 2, row = quarter * 32 + lane;
        auto sync = [] { asm volatile("bar.sync 1, 512;" ::: "memory"); };
        auto all16 = [](bool ok) -> bool {
            uint32_t r;
            asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 1, 512, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"(ok ? 1u : 0u) : "memory");
            return r != 0u;
        };
        if (tid == 0)
            for (int u = cluster; u < work.split * work.parts; u += work.clusters) tc_ticket_open(tickets + 2 * (u / work.parts) + rank, work.epoch);
        int seg = 0;
        bool ok = true;
        auto finish = [&](float (&sums)[kDnCols], const DenseToken& token, int64_t t, int64_t o0) {
            if (kGated) dn_gated<USE == kDenseGatedRows>(out, sums, t, o0, ring + (uint32_t)(kDnStages * kDnStage + warp * kDnBlock), lane);
            else dn_finish<USE>(out, token, sums, t, o0);
        };
        while (ok && walk.step(work)) {
            int m, n;
            dn_place(work, walk.tile, m, n);
            const int64_t t = (int64_t)m * kDnM + rank * 128 + row, o0 = (int64_t)n * kDnN + part * kDnCols;
            const DenseToken token = dn_token<USE>(out, t);
            float z[kDnCols];
#pragma unroll
            for (int i = 0; i < kDnCols; ++i) z[i] = 0.0f;
            for (int k = walk.k0; k < walk.k1; k += work.segment, ++seg) {
                const int buf = seg & 1;
                ok = __all_sync(kFull, tc_wait(smem_u32(&s_acc_full[buf]), (uint32_t)(seg >> 1) & 1u));
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t src = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * kDnN + part * kDnCols);
#pragma unroll
                for (int c = 0; c < kDnCols / 16; ++c) {
                    uint32_t v[16];
                    dn_read16(src + (uint32_t)(16 * c), v);
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[16 * c + i] += __uint_as_float(v[i]);
                }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0)
                    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(dn_first_sm(smem_u32(&s_acc_empty[buf]))) : "memory");
            }
            if (!(ok = all16(ok))) break;
            if (walk.k0 == 0 && walk.k1 == work.per_tile) {
                finish(z, token, t, o0);
                continue;
            }
            // a part of a tile
            constexpr int64_t slab = 128 * kDnN;
            auto slab_of = [&](int unit) { return parts + (int64_t)(2 * unit + rank) * slab + part * kDnCols * 128 + row; };
            float* const mine = slab_of(walk.unit);
#pragma unroll
            for (int k = 0; k < kDnCols; ++k) __stcg(mine + k * 128, z[k]);
            __threadfence();
            sync();
            if (tid == 0) {
                unsigned long long* const cell = tickets + 2 * walk.tile + rank;
                s_last = (int)(atomicAdd(cell, 1ull) & 255ull) == work.parts - 1;
                if (s_last) *cell = 0ull;
            }
            sync();
            if (!s_last) continue;
            __threadfence();
#pragma unroll
            for (int k = 0; k < kDnCols; ++k) z[k] = 0.0f;
            for (int i = 0; i < work.parts; ++i) {
                const float* const p = slab_of(walk.tile * work.parts + i);
#pragma unroll
                for (int k = 0; k < kDnCols; ++k) z[k] += __ldcg(p + k * 128);
            }
            finish(z, token, t, o0);
        }
        if (!ok && lane == 0) s_fail = 1;
    }
    // Every loop above is bounded, so every warp of both SMs gets here.
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (s_fail) {
        if (tid == 0) atomicExch(status, 1);
        tc_settle();
    }
    __syncwarp();
    dn_cluster_sync();  // nothing of this SM's memory is asked for any more by the other
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == kDnIssue)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * kDnN) : "memory");
}

// ---------------------------------------------------------------- host side

namespace {

struct DensePlan {
    DenseWork work{};
    size_t parts = 0, total = 0;  // byte offset (the tickets are at 0), and the bytes of all
};
// False: too large for 32-bit numbers of k-blocks.
bool dense_plan(int64_t tokens, int64_t n, int64_t k, DensePlan* p)
{
    const int64_t tm = (tokens + kDnM - 1) / kDnM, tn = (n + kDnN - 1) / kDnN, per = (k + kDnK - 1) / kDnK, tiles = tm * tn;
    if (tokens > 0x7fffff00 || n > 0x7fffff00 || k > 0x7fffff00 || tiles > 0x3fffffff / kDnGroup) return false;
    DenseWork& w = p->work;
    w.tiles_m = (int)tm;
    w.tiles_n = (int)tn;
    w.per_tile = (int)per;
    const int64_t left = tiles % kDnClusters;
    int64_t parts = left ? kDnClusters / left : 1;
    if (parts > kDnMaxParts) parts = kDnMaxParts;
    // a k-block takes 0.27 us, a part's sums 2.5 and those of the first two 6 more
    while (parts > 1 && per < 10 * parts * parts) --parts;
    if (per < 96) parts = 1;
    w.parts = (int)parts;
    w.split = parts > 1 ? (int)left : 0;
    const int64_t units = tiles + w.split * (parts - 1);
    w.clusters = (int)(units < kDnClusters ? units : kDnClusters);
    p->parts = up256((size_t)w.split * 16);
    p->total = p->parts + (size_t)w.split * w.parts * 2 * 128 * kDnN * 4;
    return true;
}

// A matrix map as tc_make_map makes, of gate and up rows in turn: the box holds 64 of each.
int dense_pair_map(const char* who, const void* b, int64_t k, int64_t ffn, CUtensorMap* map)
{
    return tc_make_map3(who, b, 2, k, 2, ffn, ffn * k * 2, k * 2, 128, 2, 64, map);
}

}  // namespace

size_t dense_ws_bytes(int64_t tokens, int64_t n, int64_t k)
{
    DensePlan p;
    return dense_plan(tokens, n, k, &p) ? p.total + 256 : 0;
}

size_t dense_ws_most() { return up256((size_t)kDnClusters * 16) + (size_t)kDnClusters * 2 * 128 * kDnN * 4; }

int dense_product(const char* who, const DenseProduct& q, const DenseOut& out, int* status, void* ws, size_t ws_bytes, cudaStream_t st)
{
    DensePlan p;
    if (!dense_plan(out.tokens, q.n, q.k, &p)) {
        set_error("%s: matrix or batch too large", who);
        return BOF4_ERR_SHAPE;
    }
    if (ws_bytes < p.total) {
        set_error("%s: the workspace has %zu bytes, %zu are needed", who, ws_bytes, p.total);
        return BOF4_ERR_WORKSPACE;
    }
    p.work.epoch = tc_next_epoch();
    p.work.segment = q.use == kDenseLoss || (q.use == kDenseGated && !out.y_bf16) ? 16 : q.use == kDenseStore ? 32 : 64;
    unsigned char* const base = static_cast<unsigned char*>(ws);
    CUtensorMap a_map, b_map;
    int rc;
    if ((rc = tc_make_map(who, q.a, 2, q.k, out.tokens, q.lda * 2, 128, 128, &a_map))) return rc;
    const int64_t ldb = q.ldb ? q.ldb : q.n_major ? q.n : q.k;
    if (q.use == kDenseGated) rc = dense_pair_map(who, q.b, q.k, q.n / 2, &b_map);
    else if (q.n_major) rc = tc_make_map(who, q.b, 2, q.n, q.k, ldb * 2, 128, kDnK, &b_map);
    else rc = tc_make_map(who, q.b, 2, q.k, q.n, ldb * 2, 128, 128, &b_map);
    if (rc) return rc;
#define BOF4_DN_GO(USE_, NMAJOR_)                                                                                                          \
    {                                                                                                                                      \
        constexpr auto kern = dense_kernel<USE_, NMAJOR_>;                                                                                 \
        if ((rc = ensure_dynamic_smem<kern>(kDnSmem))) return rc;                                                                          \
        launch_after(kern, 2 * p.work.clusters, kDnThreads, kDnSmem, st, a_map, b_map, out, status, p.work,                                \
                     reinterpret_cast<unsigned long long*>(base), reinterpret_cast<float*>(base + p.parts));                               \
    }
    const bool rows = q.use == kDenseGated && (out.align < 32 || (out.pre && out.pre_align < 32));
    if (rows) BOF4_DN_GO(kDenseGatedRows, false)
    else if (q.use == kDenseGated) BOF4_DN_GO(kDenseGated, false)
    else if (q.use == kDenseLoss) BOF4_DN_GO(kDenseLoss, false)
    else if (q.use == kDenseAdd) BOF4_DN_GO(kDenseAdd, true)
    else BOF4_DN_GO(kDenseStore, true)
#undef BOF4_DN_GO
    BOF4_CUDA_TRY(cudaGetLastError());
    return BOF4_OK;
}

}  // namespace bof4
