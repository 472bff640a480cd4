// A whole mixture-of-experts layer for a few tokens, in one launch: router, choice of experts, gated products with the 4-bit
// matrices of the chosen experts, weighted sum.
//
//   s[t, e] = sum_c x[t, c] R[e, c];  p = softmax_e(s) or sigmoid(s);  the top_k experts of a token by s (ties: lowest index)
//   h = act(G_e x) * (U_e x);  y[t] = sum_j weight[t, j] * D_e(j) h
//
// W^ as in bof4_linear: constant * level rounded to bf16.  h is kept as the sum of two bf16 values (16 bits of it reach the
// product, 2^-17 relative), everything else is fp32.
//
// With a few tokens the layer is bound by reading the codes of the experts that were chosen, once.  One cooperative launch of
// a CTA per SM goes through four phases with a barrier over the grid between them (2 us each, of which the slowest CTA's drain
// is a part; a launch of their own would cost more, and would have to build the table of level pairs anew):
//
//   router   a job per expert and four tokens, its columns over several warps; 4 us for 64 experts of 2048 columns
//   gate/up  every CTA works the choice out for itself (a warp per token), then lists the chosen experts with their tokens; 3 us.
//            Units of eight rows of G with the same eight of U (one 16-row product of decode.cuh, so that a lane holds
//            both halves of h) are dealt in equal contiguous runs over the row groups of the grid
//   down     units of 16 rows of D, the two halves of h as separate columns of the product
//   sum      y[t] over the token's experts, in the order of its list
//
// A unit's columns are split over the stripes of a row group (a warp each, 256 columns; several stripes a warp where a row is
// longer than a CTA has warps for) and its parts are added up in shared memory in a fixed order: no sum depends on scheduling.
//
// One token, 64 experts of 2048 x 1408, six chosen: 33 us, mostly latency.  19 tokens, 128 experts of 2048 x 768, eight chosen: 140 us,
// 1720 GB/s, of them router and its barrier 11, choice and list 6, gate/up 68, down 33, two barriers with the waiting for the slowest CTA
// 12, sums 2.  The walks are bound by decoding (decode.cuh), 15 to 16 codes per clock and SM.  All 128 registers a thread are taken and two spill
// (six to nine with blocks of 32).
//
// The waits on the barrier are bounded: a time-out sets the status word and everybody leaves.
#include <type_traits>

#include "decode.cuh"
#include "linear.cuh"
#include "tc.cuh"

namespace bof4 {

constexpr int kMoeWarps = 16, kMoeThreads = 32 * kMoeWarps;
constexpr int kMoeTokens = 64, kMoeExperts = 512, kMoeTop = 16;
constexpr int kMoePitch = 20;      // sums of a column, 16 rows, and room that keeps the columns of a quad in different banks
constexpr int kMoeWait = 16;       // columns of a row group that wait for the addition over the stripes
constexpr int kMoeRing = kMoeWarps * kFewSlots * kFewUnit;
constexpr int kMoeRoom = kMoeWait * kMoePitch;               // sums of a warp: of as many columns
constexpr int kMoeSums = 2 * kMoeWarps * kMoeRoom * 4;       // two buffers of them, [warp][column][row]; or the router's partial sums
constexpr int kMoeUnread = 256;    // bytes before the table that are written and not read
static_assert(kMoeSums + 20480 + kMoeUnread <= (int)kFewTable, "the sums lie before the table, behind 20 KiB of other variables");
static_assert((kMoeExperts * (kMoeTokens / 4) / kSMs + 1) * kMoeWarps * 16 <= kMoeSums, "router");
constexpr int kMoeBegin = 17408;   // dynamic memory begins there or later (behind 16.6 KiB of other variables)
constexpr int kMoeSmem = (int)kFewRing + kMoeRing - kMoeBegin;
constexpr int kMoeChoices = kMoeTokens * kMoeTop;
constexpr uint32_t kMoeSpin = 1u << 22;

struct MoeArgs {
    const uint16_t* x;
    int64_t ldx, hidden, ffn;
    int tokens, experts, top, score, act, block_shift;
    bool renormalize, router_bf16, y_bf16;
    float scale;
    const void* router;
    const void *scales1, *scales2;  // of gate and up [experts][2 ffn][hidden], of down [experts][hidden][ffn]
    const float* levels;
    void* y;
    int64_t ldy;
    int32_t* ids;
    float* weights;
    int* status;
    unsigned long long* cell;   // arrivals at the barriers in the low 16 bits, the launch's epoch above
    unsigned long long epoch;
    float* logits;              // [tokens][experts]
    uint16_t *h_hi, *h_lo;      // [tokens * top][ffn]
    float* out;                 // [tokens * top][hidden]
};

__device__ __forceinline__ float moe_sum(float v)
{
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}
// Order-preserving map of a finite or infinite fp32 value to an unsigned integer (a NaN goes to one end).
__device__ __forceinline__ uint32_t moe_key(float v)
{
    const uint32_t b = __float_as_uint(v + 0.0f);  // -0 counts as +0
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float moe_unkey(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); }

template <class ST, bool HALF>
__global__ void __launch_bounds__(kMoeThreads, 1)
moe_kernel(const __grid_constant__ CUtensorMap map1, const __grid_constant__ CUtensorMap map2, const __grid_constant__ MoeArgs p)
{
    extern __shared__ unsigned char s_dyn[];
    // the sums, the table at kFewTable, the ring
    float2* const s_pairs = reinterpret_cast<float2*>(s_dyn - smem_u32(s_dyn) + kFewTable);
    float* const s_part = reinterpret_cast<float*>(s_dyn);
    __shared__ __align__(16) float2 s_levels[8];
    __shared__ __align__(8) unsigned long long s_full[kMoeWarps][kFewSlots];
    __shared__ int2 s_what[2][kMoeWarps][kMoeWait];  // of the columns whose parts wait, by row group: tile of rows, choice
    __shared__ __align__(16) uint16_t s_id[kMoeChoices];  // expert of choice t * top + j
    __shared__ uint16_t s_list[kMoeChoices];     // choices, by expert
    __shared__ int s_count[kMoeExperts];         // choices of an expert, then its first place in the list
    __shared__ uint16_t s_first[kMoeExperts + 1], s_expert[kMoeExperts];  // of the chosen experts: first place in the list, which
    __shared__ int s_units[2][kMoeExperts + 1];  // units before a chosen expert, gate/up and down
    __shared__ int s_warp[2][kMoeWarps + 1];
    __shared__ int s_chosen, s_fail;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
    const int grid = (int)gridDim.x;
    const uint32_t column = (uint32_t)lane * 8u + kFewTable;
    if (lane < kFewSlots) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_u32(&s_full[warp][lane])) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (smem_u32(s_dyn) < (uint32_t)kMoeBegin || smem_u32(s_dyn) + kMoeSums + kMoeUnread > kFewTable) {  // not the layout that this was built for: the same for all CTAs
        if (tid == 0 && blockIdx.x == 0) *p.status = 1;
        return;
    }
    if (tid == 0) {
        s_fail = 0;
        if (blockIdx.x == 0) *p.status = 0;
    }
    if (tid == kMoeThreads - 32) {  // (a warp that mostly has nothing to do at first)
        // the cell needs no preparation: every CTA makes sure that it carries this launch's epoch before it arrives
        unsigned long long old = *reinterpret_cast<volatile unsigned long long*>(p.cell);
        while ((old & ~0xffffull) != p.epoch) {
            const unsigned long long seen = atomicCAS(p.cell, old, p.epoch);
            if (seen == old) break;
            old = seen;  // somebody else opened it or arrived: at most as many rounds as CTAs
        }
    }
    // All CTAs of the grid meet for the which-th time; false: a time-out.  What they wrote before is visible after.
    auto meet = [&](int which) -> bool {
        __threadfence();
        __syncthreads();
        if (tid == 0) {
            atomicAdd(p.cell, 1ull);
            const unsigned long long all = p.epoch + (unsigned long long)((which + 1) * grid);
            uint32_t spin = 0;
            while (*reinterpret_cast<volatile unsigned long long*>(p.cell) < all && ++spin < kMoeSpin) __nanosleep(20);
            if (spin >= kMoeSpin) {
                s_fail = 1;
                atomicExch(p.status, 1);
            }
        }
        __syncthreads();
        __threadfence();
        return s_fail == 0;
    };

    // ---- router: an expert and four tokens a job, its columns over `wide` warps
    for (int e = tid; e < p.experts; e += kMoeThreads) s_count[e] = 0;
    {
        const int quads = (p.tokens + 3) / 4, jobs = p.experts * quads, mine = jobs > (int)blockIdx.x ? (jobs - 1 - (int)blockIdx.x) / grid + 1 : 0;
        int wide = 1;
        while (wide < kMoeWarps && wide * 256 < p.hidden) wide *= 2;
        const int at_once = kMoeWarps / wide, part = warp & (wide - 1);
        for (int k = warp / wide; k < mine; k += at_once) {
            const int job = (int)blockIdx.x + k * grid, e = job / quads, t0 = (job - e * quads) * 4, n = min(4, p.tokens - t0);
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
            for (int64_t c = part * 256 + lane * 8; c < p.hidden; c += wide * 256) {
                float r[8];
                if (p.router_bf16) {
                    const uint4 u = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.router) + e * p.hidden + c));
                    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                    for (int v = 0; v < 4; ++v) r[2 * v] = __uint_as_float(w[v] << 16), r[2 * v + 1] = __uint_as_float(w[v] & 0xffff0000u);
                } else {
                    const float4* f = reinterpret_cast<const float4*>(static_cast<const float*>(p.router) + e * p.hidden + c);
                    const float4 a = __ldg(f), b = __ldg(f + 1);
                    r[0] = a.x, r[1] = a.y, r[2] = a.z, r[3] = a.w, r[4] = b.x, r[5] = b.y, r[6] = b.z, r[7] = b.w;
                }
                uint4 u[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) u[t] = t < n ? __ldg(reinterpret_cast<const uint4*>(p.x + (t0 + t) * p.ldx + c)) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const uint32_t w[4] = {u[t].x, u[t].y, u[t].z, u[t].w};
                    // (a token that is not there is left out: its zeros would make a NaN of an infinite weight)
                    if (t < n) {
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            sum[t] = fmaf(r[2 * v], __uint_as_float(w[v] << 16), sum[t]);
                            sum[t] = fmaf(r[2 * v + 1], __uint_as_float(w[v] & 0xffff0000u), sum[t]);
                        }
                    }
                }
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) sum[t] = moe_sum(sum[t]);
            if (lane == 0) *reinterpret_cast<float4*>(s_part + (k * kMoeWarps + part) * 4) = make_float4(sum[0], sum[1], sum[2], sum[3]);
        }
        __syncthreads();
        for (int i = tid; i < mine * 4; i += kMoeThreads) {
            const int k = i >> 2, job = (int)blockIdx.x + k * grid, e = job / quads, t = (job - e * quads) * 4 + (i & 3);
            float sum = 0.0f;
            for (int w = 0; w < wide; ++w) sum += s_part[(k * kMoeWarps + w) * 4 + (i & 3)];
            if (t < p.tokens) p.logits[t * p.experts + e] = sum;
        }
    }
    if (tid < 8) s_levels[tid] = make_float2(__ldg(p.levels + 2 * tid), __ldg(p.levels + 2 * tid + 1));
    fill_pairs(s_pairs, p.levels, tid, kMoeThreads);
    if (!meet(0)) return;

    // ---- the choice, by every CTA for itself
    const int ranks = (p.experts + 31) / 32;  // experts of a lane
    for (int t = warp; t < p.tokens; t += kMoeWarps) {
        constexpr int R = kMoeExperts / 32;
        float s[R];
        float most = -INFINITY;
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (k >= ranks) break;
            const int e = k * 32 + lane;
            s[k] = e < p.experts ? __ldcg(p.logits + t * p.experts + e) : 0.0f;
        }
        float total = 0.0f;
        if (p.score == BOF4_SCORE_SOFTMAX) {
#pragma unroll
            for (int k = 0; k < R; ++k) {
                if (k >= ranks) break;
                if (k * 32 + lane < p.experts) most = fmaxf(most, s[k]);
            }
#pragma unroll
            for (int o = 16; o >= 1; o >>= 1) most = fmaxf(most, __shfl_xor_sync(kFull, most, o));
#pragma unroll
            for (int k = 0; k < R; ++k) {
                if (k >= ranks) break;
                if (k * 32 + lane < p.experts) total += expf(s[k] - most);
            }
            total = moe_sum(total);
        }
        // the lane's experts as keys, 0 for one that is taken, and the first of its largest ones: only the lane whose expert is taken
        // looks for its next one
        uint32_t key[R], best = 0u, which = 0u;
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (k >= ranks) break;
            const int e = k * 32 + lane;
            key[k] = e < p.experts ? max(moe_key(s[k]), 1u) : 0u;
            if (key[k] > best) best = key[k], which = (uint32_t)e;
        }
        float mine = 0.0f;  // lane j: the logit of choice j, then its score
        int chosen_e = 0;   // and which it is
        for (int j = 0; j < p.top; ++j) {
            // the largest remaining logit, then the lowest index
            const uint32_t top = __reduce_max_sync(kFull, best), e = __reduce_min_sync(kFull, best == top ? which : 0xffffffffu);
            if (lane == j) mine = moe_unkey(top), chosen_e = (int)e;
            if ((e & 31u) == (uint32_t)lane) {
                best = 0u;
#pragma unroll
                for (int k = 0; k < R; ++k) {
                    if (k >= ranks) break;
                    if ((uint32_t)k == e >> 5) key[k] = 0u;
                    if (key[k] > best) best = key[k], which = (uint32_t)(k * 32 + lane);
                }
            }
        }
        // Scores that are divided by their sum may have a common factor: where the token's largest logit `lead` is negative the logistic ones
        // are exp(l) / (1 + exp(l)) with exp(lead) taken out, so that the largest is at least 1/2.  (1 / (1 + exp(-l)) is 0 for l < -88.7.)
        const float lead = p.score == BOF4_SCORE_SIGMOID && p.renormalize ? fminf(__shfl_sync(kFull, mine, 0), 0.0f) : 0.0f;
        if (lane >= p.top) mine = 0.0f;
        else if (p.score == BOF4_SCORE_SOFTMAX) mine = expf(mine - most) / total;
        else if (lead < 0.0f) mine = expf(mine - lead) / (1.0f + expf(mine));
        else mine = 1.0f / (1.0f + expf(-mine));
        if (p.renormalize) mine /= moe_sum(mine);
        if (lane < p.top) {
            const int a = t * p.top + lane;
            s_id[a] = (uint16_t)chosen_e;
            atomicAdd(&s_count[chosen_e], 1);
            if (blockIdx.x == 0) p.ids[a] = chosen_e, p.weights[a] = mine * p.scale;
        }
    }
    __syncthreads();
    // ---- the chosen experts in ascending order, their choices, and the units before each
    const int choices = p.tokens * p.top;
    const int tiles1 = (int)(p.ffn / 8), tiles2 = (int)(p.hidden / 16);
    {
        const int count = tid < p.experts ? s_count[tid] : 0;
        // running numbers over the threads: choices, and chosen experts
        int before = count, which = count > 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int b = __shfl_up_sync(kFull, before, o), w = __shfl_up_sync(kFull, which, o);
            if (lane >= o) before += b, which += w;
        }
        if (lane == 31) s_warp[0][warp] = before, s_warp[1][warp] = which;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kMoeWarps; ++w)
            if (w < warp) before += s_warp[0][w], which += s_warp[1][w];
        if (count > 0) {
            const int i = which - 1;
            s_expert[i] = (uint16_t)tid;
            s_first[i] = (uint16_t)(before - count);
            s_count[tid] = before - count;
            // passes of eight tokens (gate/up) and of four (down)
            s_units[0][i] = (count + 7) / 8 * tiles1;
            s_units[1][i] = (count + 3) / 4 * tiles2;
        }
        if (tid == kMoeThreads - 1) s_chosen = which, s_first[which] = (uint16_t)choices;
    }
    __syncthreads();
    // a choice's place in its expert's list: the choices before it with the same expert.  (All CTAs need the same order: an expert's
    // passes take their tokens from it.)
    for (int a = tid; a < choices; a += kMoeThreads) {
        const uint32_t id = s_id[a], twice = id << 16 | id;
        int rank = 0;
        for (int b = 0; b < a; b += 8) {
            const uint4 v = *reinterpret_cast<const uint4*>(s_id + b);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t x = w[k] ^ twice;
                rank += (b + 2 * k < a && (x & 0xffffu) == 0u) + (b + 2 * k + 1 < a && (x >> 16) == 0u);
            }
        }
        s_list[s_count[id] + rank] = (uint16_t)a;
    }
    const int chosen = s_chosen;
    if (warp < 2) {  // exclusive sums over the chosen experts, by a warp each
        int carry = 0;
        for (int i0 = 0; i0 < chosen; i0 += 32) {
            const int i = i0 + lane, v = i < chosen ? s_units[warp][i] : 0;
            int sum = v;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int b = __shfl_up_sync(kFull, sum, o);
                if (lane >= o) sum += b;
            }
            if (i < chosen) s_units[warp][i] = carry + sum - v;
            carry += __shfl_sync(kFull, sum, 31);
        }
        if (lane == 0) s_units[warp][chosen] = carry;
    }
    __syncthreads();

    // ---- gate/up and down: the same walk over units
    int slot = 0;            // of the ring, over both walks: nothing is on its way between them
    uint32_t parity = 0;
    bool failed = false;     // a wait for codes ran out
    const uint32_t ring = kFewRing + (uint32_t)(warp * kFewSlots * kFewUnit);
    // `before`: what has to happen before the first tokens are read; codes are on their way by then.  False: it failed.
    auto walk = [&](auto second_c, auto&& before) -> bool {
        constexpr bool SECOND = decltype(second_c)::value;
        constexpr int PASS = SECOND ? 4 : 8;
        const int* const units = s_units[SECOND ? 1 : 0];
        const int cols = (int)(SECOND ? p.ffn : p.hidden), hidden = (int)p.hidden, ffn = (int)p.ffn, tiles = SECOND ? tiles2 : tiles1;
        const void* const scales = SECOND ? p.scales2 : p.scales1;
        const int per_row = cols >> p.block_shift;
        const int stripes = (cols + kFewStripe - 1) / kFewStripe, rounds = (stripes + kMoeWarps - 1) / kMoeWarps;
        const int wide = (stripes + rounds - 1) / rounds, groups = kMoeWarps / wide;  // stripes side by side, row groups of the CTA
        const int group = warp / wide, stripe = warp - group * wide;
        const bool busy = group < groups;
        const int total = units[chosen], all = grid * groups, each = total / all, extra = total % all;
        auto start_of = [&](int k) { return k * each + min(k, extra); };  // first unit of row group k of the grid
        const int group0 = (int)blockIdx.x * groups;
        const int begin = busy ? start_of(group0 + group) : 0, mine = busy ? start_of(group0 + group + 1) - begin : 0;
        // a place in the order of units: expert (of the chosen ones), pass over its tokens, tile of its rows, round over the stripes
        struct Place {
            int i, pass, tile, round;
        };
        auto columns_of = [&](const Place& u) { return s_first[u.i + 1] - s_first[u.i] - u.pass * PASS; };  // tokens left for the pass
        auto step_on = [&](Place& u) {
            if (++u.round < rounds) return;
            u.round = 0;
            if (++u.tile < tiles) return;
            u.tile = 0;
            if (columns_of(u) > PASS) ++u.pass;
            else ++u.i, u.pass = 0;
        };
        Place now{0, 0, 0, 0};
        if (mine) {
            while (begin >= units[now.i + 1]) ++now.i;
            const int in = begin - units[now.i];
            now.pass = in / tiles, now.tile = in - now.pass * tiles;
        }
        Place ask = now;
        int asked = 0, row0 = 0, row1 = 0;   // rows of the unit that is asked for next, first of its eight and of the other eight
        int64_t at0 = 0, at1 = 0;            // the lane's constants in rows g of each
        auto aim = [&] {
            const int e = s_expert[ask.i], cc = (ask.round * wide + stripe) * kFewStripe + 64 * q;
            row0 = SECOND ? e * hidden + ask.tile * 16 : e * 2 * ffn + ask.tile * 8;
            row1 = SECOND ? row0 + 8 : row0 + ffn;
            at0 = (int64_t)(row0 + g) * per_row + (cc >> p.block_shift);
            at1 = (int64_t)(row1 + g) * per_row + (cc >> p.block_shift);
        };
        if (mine) aim();
        FewConst<ST, HALF> m[kFewAhead + 1];
        auto request = [&](int k, FewConst<ST, HALF>& c) {
            const bool ok = asked < mine * rounds;
            const int c0 = (ask.round * wide + stripe) * kFewStripe, cc = c0 + 64 * q;
            if (ok && lane == 0 && !failed) {
                const uint32_t bar = smem_u32(&s_full[warp][k]), dst = ring + (uint32_t)(k * kFewUnit);
                asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"((uint32_t)kFewUnit) : "memory");
#pragma unroll
                for (int h = 0; h < (SECOND ? 1 : 2); ++h)
                    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                                 :
                                 : "r"(dst + h * 1024u), "l"(reinterpret_cast<uint64_t>(SECOND ? &map2 : &map1)), "r"(bar), "r"(c0 >> 1), "r"(h ? row1 : row0)
                                 : "memory");
            }
            c.load(scales, at0, at1, (ok && cc < cols ? 5u : 0u) | (ok && cc + 32 < cols ? 10u : 0u));
            ++asked;
            if (!ok) return;
            step_on(ask);
            if (asked == mine * rounds) return;
            if (rounds == 1 && ask.tile) {  // the next rows of the same expert
                constexpr int next = SECOND ? 16 : 8;
                row0 += next, row1 += next;
                at0 += next * per_row, at1 += next * per_row;
            } else {
                aim();
            }
        };
        // (ring slots go on from where the walk before ended)
        auto slot_after = [&](int k) { return slot + k >= kFewSlots ? slot + k - kFewSlots : slot + k; };
#pragma unroll
        for (int k = 0; k < kFewAhead; ++k) request(slot_after(k), m[k]);
        if (!before()) {  // nothing of this CTA may be on its way when it ends
            for (int k = 0; k < min(asked, mine * rounds); ++k)
                if (k < kFewAhead && !failed) (void)tc_wait(smem_u32(&s_full[warp][slot_after(k)]), slot + k >= kFewSlots ? parity ^ 1u : parity);
            return false;
        }
        // Sums of a unit's columns wait until no room is left for those of the next one; then the stripes of the row group meet and add them
        // up.  (Row groups have their own barriers and cadence.  With one of the whole CTA, at places that suited the unit with the most
        // columns it took longer.)
        int cols_waiting = 0, buf = 0, have_i = -1, have_pass = -1;  // whose tokens xr holds
        uint32_t xr[1][32];
        for (int s = 0; s < mine; ++s) {
            float acc[1][4] = {};
            const int columns = min(columns_of(now), PASS), place = s_first[now.i] + now.pass * PASS;
            if (stripe == 0 && lane < columns) s_what[buf][group][cols_waiting + lane] = make_int2(now.tile, s_list[place + lane]);
            for (int round = 0; round < rounds; ++round) {
                __syncwarp();  // all lanes have read the slot that is asked for now
                request(slot_after(kFewAhead), m[kFewAhead]);
                if (rounds > 1 || now.i != have_i || now.pass != have_pass) {
                    have_i = now.i, have_pass = now.pass;
                    const int c0 = (round * wide + stripe) * kFewStripe + 64 * q, col = SECOND ? g & 3 : g;
                    const bool live = col < columns;
                    const int a = live ? s_list[place + col] : 0;
                    const uint16_t* src = SECOND ? (g < 4 ? p.h_hi : p.h_lo) + (int64_t)a * ffn : p.x + (int64_t)(a / p.top) * p.ldx;
                    few_tokens(xr[0], src + c0, live && c0 < cols, live && c0 + 32 < cols);
                }
                if (!failed && !tc_wait(smem_u32(&s_full[warp][slot]), parity)) failed = true;
                FewCodes code;
                few_read(code, ring + (uint32_t)(slot * kFewUnit), lane);
                few_multiply<ST, HALF, 1>(code, m[0], xr, acc, column, s_levels);
                // The slot is asked for again in the next round: by then its codes have to be in registers, not only their loads under way.
                // A sum of this round depends on all of them, so it is stored, where nobody reads it.  (The last round's sums are stored below.)
                if (rounds > 1) asm volatile("st.shared.f32 [%0], %1;" ::"r"(column - kMoeUnread), "f"(acc[0][0]) : "memory");
                if (++slot == kFewSlots) slot = 0, parity ^= 1u;
#pragma unroll
                for (int u = 0; u < kFewAhead; ++u) m[u] = m[u + 1];
                step_on(now);
            }
            if (SECOND) {
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[0][v] += __shfl_xor_sync(kFull, acc[0][v], 2);  // columns c and c + 4: the two halves of h
            }
            float* const to = s_part + (buf * kMoeWarps + warp) * kMoeRoom + (cols_waiting + 2 * q) * kMoePitch + g;
            if (2 * q < columns) to[0] = acc[0][0], to[8] = acc[0][2];
            if (2 * q + 1 < columns) to[kMoePitch] = acc[0][1], to[kMoePitch + 8] = acc[0][3];
            cols_waiting += columns;
            if (s + 1 < mine && cols_waiting + min(columns_of(now), PASS) <= kMoeWait) continue;
            if (wide > 1) asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(wide * 32) : "memory");
            else __syncwarp();
            // rows along the lanes
            constexpr int ROWS = SECOND ? 16 : 8;
            for (int e = stripe * 32 + lane; e < cols_waiting * ROWS; e += wide * 32) {
                const int row = e % ROWS, col = e / ROWS;
                const int2 what = s_what[buf][group][col];
                const float* part = s_part + (buf * kMoeWarps + group * wide) * kMoeRoom + col * kMoePitch + row;
                float v0 = 0.0f, v1 = 0.0f;
#pragma unroll 4
                for (int w = 0; w < wide; ++w) {
                    v0 += part[w * kMoeRoom];
                    if (!SECOND) v1 += part[w * kMoeRoom + 8];
                }
                if (SECOND) {
                    p.out[(int64_t)what.y * hidden + what.x * 16 + row] = v0;
                } else {
                    const float h = activate(v0, p.act) * v1;
                    uint16_t hi = bf16_round(h);
                    if (isfinite(h) && (hi & 0x7fffu) == 0x7f80u) --hi;  // above the largest bf16 value: that one, and the rest in the second half
                    const int64_t o = (int64_t)what.y * ffn + what.x * 8 + row;
                    p.h_hi[o] = hi;
                    p.h_lo[o] = bf16_round(isfinite(h) ? h - bf16_value(hi) : 0.0f);
                }
            }
            buf ^= 1;
            cols_waiting = 0;
        }
        if (failed) {  // nothing was asked for since; what was before must not reach shared memory after the CTA has left
            atomicExch(p.status, 1);
            tc_settle();
        }
        return true;
    };
    if (!walk(std::false_type{}, [] { return true; })) return;
    if (!walk(std::true_type{}, [&] { return meet(1); })) return;
    if (!meet(2)) return;

    // ---- the weighted sums
    for (int64_t i = (int64_t)blockIdx.x * kMoeThreads + tid; i < p.tokens * p.hidden; i += (int64_t)grid * kMoeThreads) {
        const int64_t t = i / p.hidden, o = i - t * p.hidden;
        float sum = 0.0f;
        for (int j = 0; j < p.top; ++j) sum = fmaf(__ldcg(p.weights + t * p.top + j), __ldcg(p.out + (t * p.top + j) * p.hidden + o), sum);
        if (p.y_bf16) static_cast<uint16_t*>(p.y)[t * p.ldy + o] = bf16_round(sum);
        else static_cast<float*>(p.y)[t * p.ldy + o] = sum;
    }
    // the last to leave clears the cell: a replayed launch has the same epoch
    if (tid == 0 && (int)(atomicAdd(p.cell, 1ull) & 0xffffull) == 4 * grid - 1) *p.cell = 0ull;
}

namespace {

struct MoePlan {
    size_t logits, hi, lo, out, total;  // byte offsets (the barriers' cell is at 0), and the bytes of all
};
MoePlan moe_plan(int64_t tokens, int64_t hidden, int64_t ffn, int64_t experts, int64_t top)
{
    MoePlan p;
    p.logits = 256;
    p.hi = p.logits + up256((size_t)(tokens * experts * 4));
    p.lo = p.hi + up256((size_t)(tokens * top * ffn * 2));
    p.out = p.lo + up256((size_t)(tokens * top * ffn * 2));
    p.total = p.out + up256((size_t)(tokens * top * hidden * 4));
    return p;
}
bool moe_sizes(int64_t tokens, int64_t hidden, int64_t ffn, int64_t experts, int64_t top)
{
    return tokens >= 0 && tokens <= kMoeTokens && experts >= 1 && experts <= kMoeExperts && top >= 1 && top <= kMoeTop && top <= experts && hidden >= 32 &&
           hidden <= (1 << 20) && ffn >= 32 && ffn <= (1 << 20) && hidden % 32 == 0 && ffn % 32 == 0;
}

}  // namespace
}  // namespace bof4

using namespace bof4;

extern "C" size_t bof4_moe_workspace_bytes(int64_t n_tokens, int64_t hidden, int64_t ffn, int n_experts, int top_k)
{
    return moe_sizes(n_tokens, hidden, ffn, n_experts, top_k) ? moe_plan(n_tokens, hidden, ffn, n_experts, top_k).total : 0;
}

extern "C" int bof4_moe(const void* d_x, int64_t ldx, int64_t n_tokens, int64_t hidden, const void* d_router, int router_dtype, int n_experts,
                        int top_k, int score, int renormalize, float scale, const uint8_t* d_gate_up_codes, const void* d_gate_up_scales,
                        const uint8_t* d_down_codes, const void* d_down_scales, int scale_dtype, int64_t ffn, int block_size,
                        const float* d_codebook, int activation, void* d_y, int y_dtype, int64_t ldy, int32_t* d_ids, float* d_weights,
                        int* d_status, void* d_ws, size_t ws_bytes, void* stream)
{
    const char* fn = "bof4_moe";
    if (!moe_sizes(n_tokens, hidden, ffn, n_experts, top_k) || !valid_block_size(block_size) || hidden % block_size || ffn % block_size) {
        set_error("%s: 0 ... 64 tokens, 1 ... 512 experts, top_k 1 ... 16 and at most n_experts, block_size a power of two in 32 ... 4096 that "
                  "divides hidden and ffn (at most 2^20)", fn);
        return BOF4_ERR_SHAPE;
    }
    if ((scale_dtype != BOF4_F32 && scale_dtype != BOF4_BF16) || (router_dtype != BOF4_F32 && router_dtype != BOF4_BF16) ||
        (y_dtype != BOF4_F32 && y_dtype != BOF4_BF16)) {
        set_error("%s: unknown dtype", fn);
        return BOF4_ERR_DTYPE;
    }
    if (activation < BOF4_ACT_NONE || activation > BOF4_ACT_SILU || (score != BOF4_SCORE_SOFTMAX && score != BOF4_SCORE_SIGMOID)) {
        set_error("%s: unknown activation or score", fn);
        return BOF4_ERR_INVALID_ARG;
    }
    if (n_tokens > 1 && (ldx < hidden || ldy < hidden)) {
        set_error("%s: a row stride is smaller than its row", fn);
        return BOF4_ERR_SHAPE;
    }
    if (n_tokens <= 1) ldx = ldy = hidden;
    if (!d_status || (n_tokens > 0 && (!d_x || !d_router || !d_gate_up_codes || !d_gate_up_scales || !d_down_codes || !d_down_scales || !d_codebook ||
                                       !d_y || !d_ids || !d_weights))) {
        set_error("%s: NULL pointer", fn);
        return BOF4_ERR_INVALID_ARG;
    }
    auto odd = [](const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; };
    if (n_tokens > 0 && (odd(d_gate_up_codes, 32) || odd(d_down_codes, 32) || odd(d_x, 16) || odd(d_router, 16) || ldx % 8)) {
        set_error("%s: codes must be 32-byte aligned, d_x and d_router 16-byte aligned and ldx a multiple of 8", fn);
        return BOF4_ERR_INVALID_ARG;
    }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (n_tokens == 0) {
        BOF4_CUDA_TRY(cudaMemsetAsync(d_status, 0, sizeof(int), st));
        return BOF4_OK;
    }
    const MoePlan plan = moe_plan(n_tokens, hidden, ffn, n_experts, top_k);
    if (!d_ws || odd(d_ws, 256) || ws_bytes < plan.total) {
        set_error("%s: the workspace must be 256-byte aligned and hold %zu bytes", fn, plan.total);
        return BOF4_ERR_WORKSPACE;
    }
    unsigned char* const base = static_cast<unsigned char*>(d_ws);
    MoeArgs a{};
    a.x = static_cast<const uint16_t*>(d_x);
    a.ldx = ldx;
    a.hidden = hidden;
    a.ffn = ffn;
    a.tokens = (int)n_tokens;
    a.experts = n_experts;
    a.top = top_k;
    a.score = score;
    a.act = activation;
    while ((1 << a.block_shift) < block_size) ++a.block_shift;
    a.renormalize = renormalize != 0;
    a.router_bf16 = router_dtype == BOF4_BF16;
    a.y_bf16 = y_dtype == BOF4_BF16;
    a.scale = scale;
    a.router = d_router;
    a.scales1 = d_gate_up_scales;
    a.scales2 = d_down_scales;
    a.levels = d_codebook;
    a.y = d_y;
    a.ldy = ldy;
    a.ids = d_ids;
    a.weights = d_weights;
    a.status = d_status;
    a.cell = reinterpret_cast<unsigned long long*>(base);
    do a.epoch = tc_next_epoch() & ~0xffffull;
    while (!a.epoch);
    a.logits = reinterpret_cast<float*>(base + plan.logits);
    a.h_hi = reinterpret_cast<uint16_t*>(base + plan.hi);
    a.h_lo = reinterpret_cast<uint16_t*>(base + plan.lo);
    a.out = reinterpret_cast<float*>(base + plan.out);
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeCooperative;  // all CTAs are resident at once: they meet at barriers
    attr.val.cooperative = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(kSMs);
    cfg.blockDim = dim3(kMoeThreads);
    cfg.dynamicSmemBytes = kMoeSmem;
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int rc;
    CUtensorMap map1, map2;
    if ((rc = tc_make_map(fn, d_gate_up_codes, 1, hidden / 2, n_experts * 2 * ffn, hidden / 2, 128, 8, &map1)) ||
        (rc = tc_make_map(fn, d_down_codes, 1, ffn / 2, n_experts * hidden, ffn / 2, 128, 16, &map2)))
        return rc;
#define BOF4_MOE_GO(ST_, HALF_)                                                  \
    {                                                                            \
        constexpr auto kern = moe_kernel<ST_, HALF_>;                            \
        if ((rc = ensure_dynamic_smem<kern>(kMoeSmem))) return rc;               \
        BOF4_CUDA_TRY(cudaLaunchKernelEx(&cfg, kern, map1, map2, static_cast<MoeArgs>(a)));  \
    }
    if (scale_dtype == BOF4_F32) {
        if (block_size == 32) BOF4_MOE_GO(F32, true) else BOF4_MOE_GO(F32, false)
    } else {
        if (block_size == 32) BOF4_MOE_GO(BF16, true) else BOF4_MOE_GO(BF16, false)
    }
#undef BOF4_MOE_GO
    return BOF4_OK;
}
