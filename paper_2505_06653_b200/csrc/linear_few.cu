// bof4_linear for one to sixteen tokens: a product that is bound by its codes.
//
// A CTA holds `groups` row groups of `stripes` warps.  Warp s of a group owns 256 columns of a slice of the columns for every
// row tile (16 rows) that the group visits, its tokens in registers (decode.cuh).  The parts of a row tile are added up over
// the stripes in shared memory, in a fixed order, a few row tiles at a time (two buffers, one barrier per FewGeo::defer tiles).
// A matrix with more columns than a CTA has warps for is cut into slices of equal numbers of stripes; the CTAs of a slice
// take the same row tiles as their counterparts in the others, leave their sums in the workspace, and the one that is last
// (a ticket: nobody waits) adds the slices up in order.
//
// Bound by decoding (decode.cuh), and in small calls by set-up: the table of level pairs, the first codes and the drain take 4 us.
// 4096 x 4096 by one token 7.0 us, 11008 x 4096 by five 14.0, 28672 x 8192 by one 42 to 45, by eight 50 to 55.
#include "decode.cuh"
#include "linear.cuh"
#include "tc.cuh"

namespace bof4 {

constexpr int kFewPitch = 20;  // rows of a token, 16, and room that keeps the tokens of a quad in different banks
template <int NT>
struct FewGeo {
    // a lane keeps 32 registers of tokens per eight of them: 128 registers a thread for 8 tokens, 255 for 16
    static constexpr int warps = NT == 1 ? 16 : 8, threads = 32 * warps;
    static constexpr int ring = warps * kFewSlots * kFewUnit;
    // row tiles between two additions over the stripes: as many as two buffers of sums, [tile][warp][token][row], have room for
    // before the table (the fewer barriers the better: with two of them 28672 x 8192 by one token takes 6 us more than without any)
    static constexpr int sums = 54 * 1024;
    static int defer(int tokens)
    {
        const int d = sums / (2 * warps * tokens * kFewPitch * 4);
        return d < 16 ? d : 16;
    }
    static_assert(sums + 8192 <= (int)kFewTable, "the sums lie before the table");
};

constexpr int kFewBegin = 1024;  // dynamic memory begins there or later

struct FewWork {
    int stripes, groups, slices, peers;  // stripes of a slice; CTAs of a slice
    int tiles, defer;
    unsigned long long epoch;
};

template <int NT, class ST, bool HALF>
__global__ void __launch_bounds__(FewGeo<NT>::threads, 1)
linear_few_kernel(const __grid_constant__ CUtensorMap code_map, const void* __restrict__ scales, int64_t rows, int64_t cols, int block_shift,
                  const float* __restrict__ levels, const uint16_t* __restrict__ x, int64_t ldx, const LinearOut out,
                  const float* __restrict__ correction, int* __restrict__ status, const FewWork work, unsigned long long* __restrict__ tickets,
                  float* __restrict__ sums)
{
    if (!after_previous()) return;
    constexpr int W = FewGeo<NT>::warps;
    const int D = work.defer, P = (int)out.tokens * kFewPitch;
    extern __shared__ unsigned char s_dyn[];
    // the sums, the table at kFewTable, the ring
    unsigned char* const s_zero = s_dyn - smem_u32(s_dyn);
    float2* const s_pairs = reinterpret_cast<float2*>(s_zero + kFewTable);
    float* const s_part = reinterpret_cast<float*>(s_dyn);  // [2][D][W][P]
    __shared__ __align__(16) float2 s_levels[8];
    __shared__ __align__(8) unsigned long long s_full[W][kFewSlots];
    __shared__ int s_last;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
    const int group = warp / work.stripes, stripe = warp - group * work.stripes;
    const int slice = (int)blockIdx.x / work.peers, peer = (int)blockIdx.x - slice * work.peers;
    const int64_t c0 = (int64_t)(slice * work.stripes + stripe) * kFewStripe + 64 * q;
    const bool busy = group < work.groups, live0 = busy && c0 < cols, live1 = busy && c0 + 32 < cols;
    const int first = peer * work.groups + group, step = work.peers * work.groups;  // row tiles of this group
    const int rounds = (work.tiles - peer * work.groups + step - 1) / step;         // of the CTA: its first group has the most
    const int tokens = (int)out.tokens;
    if (smem_u32(s_dyn) < (uint32_t)kFewBegin || smem_u32(s_dyn) + FewGeo<NT>::sums > kFewTable) {  // not the layout that this was built for
        if (tid == 0 && blockIdx.x == 0) *status = 1;
        return;
    }
    bool failed = false;  // a wait ran out
    if (tid == 0) {
        if (blockIdx.x == 0) *status = 0;  // long before any wait can have run out
        if (work.slices > 1) tc_ticket_open(tickets + peer, work.epoch);
    }
    // The group's row tiles in order: codes and constants are requested kFewAhead of them before they are used.
    const uint32_t ring = kFewRing + (uint32_t)(warp * kFewSlots * kFewUnit), lanes = (live0 ? 5u : 0u) | (live1 ? 10u : 0u);
    const int mine = busy && first < work.tiles ? (work.tiles - 1 - first) / step + 1 : 0;  // row tiles of this group
    const int64_t per_row = cols >> block_shift, jump = (int64_t)step * 16 * per_row;
    int64_t at = ((int64_t)first * 16 + g) * per_row + (c0 >> block_shift);
    int left = (int)(rows - (int64_t)first * 16) - g, row = first * 16, asked = 0;
    FewConst<ST, HALF> m[kFewAhead + 1];  // of the next units, the oldest first
    auto request = [&](int slot, FewConst<ST, HALF>& c) {
        if (asked < mine && lane == 0 && !failed)
            tc_load_box(ring + (uint32_t)(slot * kFewUnit), &code_map, &s_full[warp][slot], kFewUnit, (int)(c0 >> 1), row);
        c.load(scales, at, at + 8 * per_row, ((left > 0 ? 3u : 0u) | (left > 8 ? 12u : 0u)) & lanes);
        ++asked, row += step * 16, left -= step * 16, at += jump;
    };
    if (lane < kFewSlots) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_u32(&s_full[warp][lane])) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncwarp();
#pragma unroll
    for (int k = 0; k < kFewAhead; ++k) request(k, m[k]);
    uint32_t xr[NT][32];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int t = 8 * n + g;
        few_tokens(xr[n], x + (int64_t)(t < tokens ? t : 0) * ldx + c0, live0 && t < tokens, live1 && t < tokens);
    }
    if (tid < 8) s_levels[tid] = make_float2(__ldg(levels + 2 * tid), __ldg(levels + 2 * tid + 1));
    fill_pairs(s_pairs, levels, tid, FewGeo<NT>::threads);
    __syncthreads();
    const uint32_t column = (uint32_t)lane * 8u + kFewTable;
    int k = 0, buf = 0, slot = 0;
    uint32_t parity = 0;
    for (int i = 0; i < rounds; ++i) {
        __syncwarp();  // all lanes have read the slot that is asked for now
        request(slot == 0 ? kFewAhead : slot - 1, m[kFewAhead]);
        float acc[NT][4] = {};
        if (i < mine) {
            if (!failed && !tc_wait(smem_u32(&s_full[warp][slot]), parity)) failed = true;
            FewCodes code;
            few_read(code, ring + (uint32_t)(slot * kFewUnit), lane);
            few_multiply<ST, HALF, NT>(code, m[0], xr, acc, column, s_levels);
        }
        if (++slot == kFewSlots) slot = 0, parity ^= 1u;
        float* const to0 = s_part + ((buf * D + k) * W + warp) * P + 2 * q * kFewPitch + g;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float* const to = to0 + 8 * n * kFewPitch;
            const int t = 8 * n + 2 * q;
            if (t < tokens) to[0] = acc[n][0], to[8] = acc[n][2];
            if (t + 1 < tokens) to[kFewPitch] = acc[n][1], to[kFewPitch + 8] = acc[n][3];
        }
        if (k == D - 1 || i + 1 == rounds) {
            __syncthreads();
            // the k + 1 row tiles of each group since the last time; rows along the lanes, so that neighbours write neighbours
            for (uint32_t w = (uint32_t)tid >> 4; w < (uint32_t)((k + 1) * work.groups * tokens); w += FewGeo<NT>::threads / 16) {
                const uint32_t rest = w / (uint32_t)tokens, t = w - rest * (uint32_t)tokens, j = rest / (uint32_t)work.groups, gr = rest - j * (uint32_t)work.groups;
                const int64_t r = ((int64_t)peer * work.groups + gr + (int64_t)(i - k + (int)j) * step) * 16 + (lane & 15);
                const float* p = s_part + ((buf * D + j) * W + gr * work.stripes) * P + t * kFewPitch + (lane & 15);
                if (r >= rows) continue;
                float sum = 0.0f;
#pragma unroll 8
                for (int s = 0; s < work.stripes; ++s) sum += p[s * P];
                if (work.slices > 1)
                    sums[((int64_t)slice * tokens + t) * (work.tiles * 16) + r] = sum;
                else
                    out.store(sum + (correction ? correction[(int64_t)t * rows + r] : 0.0f), out.bias_at(r), out.residual_at(t, r), t, r);
            }
            buf ^= 1;
            k = 0;
        } else {
            ++k;
        }
#pragma unroll
        for (int u = 0; u < kFewAhead; ++u) m[u] = m[u + 1];
    }
    if (failed) {  // nothing was asked for since; what was before must not reach shared memory after the CTA has left
        atomicExch(status, 1);
        tc_settle();
    }
    if (work.slices == 1) return;
    __threadfence();
    __syncthreads();
    if (tid == 0) {
        s_last = (int)(atomicAdd(tickets + peer, 1ull) & 255ull) == work.slices - 1;
        if (s_last) tickets[peer] = 0ull;
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    // four rows a thread, several slices on their way at a time
    const int64_t pitch = (int64_t)work.tiles * 16;
    for (uint32_t w = (uint32_t)tid >> 2; w < (uint32_t)(rounds * work.groups * tokens); w += FewGeo<NT>::threads / 4) {
        const uint32_t rest = w / (uint32_t)tokens, t = w - rest * (uint32_t)tokens, i = rest / (uint32_t)work.groups, gr = rest - i * (uint32_t)work.groups;
        const int64_t tile = (int64_t)peer * work.groups + gr + (int64_t)i * step, r = tile * 16 + 4 * (lane & 3);
        if (tile >= work.tiles) continue;
        const float4* p = reinterpret_cast<const float4*>(sums + (int64_t)t * pitch + r);
        const int64_t next = tokens * pitch / 4;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s = 0; s < work.slices; s += 4) {
            float4 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = s + u < work.slices ? __ldcg(p + (s + u) * next) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int u = 0; u < 4; ++u) sum.x += v[u].x, sum.y += v[u].y, sum.z += v[u].z, sum.w += v[u].w;
        }
        const float z[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (r + u < rows)
                out.store(z[u] + (correction ? correction[(int64_t)t * rows + r + u] : 0.0f), out.bias_at(r + u), out.residual_at(t, r + u), t, r + u);
    }
}

// Outliers: correction[t, r] = sum over the entries of row r of (val - W^) x[t, c], zero elsewhere (set before).  A CTA takes 256
// entries: their changes, a term per entry and token, and a row's terms added up in the order of the list; what is left of a row
// more than 64 entries behind them comes from global memory.
constexpr int kFewTokens = 16, kFewListTokens = 6;  // tokens of a call, without and with a list
template <class ST>
__device__ __forceinline__ float scale_at(const void* scales, int64_t b)
{
    return ST::code == BOF4_F32 ? __ldg(static_cast<const float*>(scales) + b) : bf16_value(__ldg(static_cast<const uint16_t*>(scales) + b));
}
template <class ST>
__global__ void __launch_bounds__(256)
few_correction_kernel(const uint8_t* __restrict__ codes, const void* __restrict__ scales, int64_t rows, int64_t cols, int block_shift,
                      const float* __restrict__ levels, const uint16_t* __restrict__ x, int64_t ldx, int tokens, const int32_t* __restrict__ idx,
                      const uint16_t* __restrict__ val, const int64_t* __restrict__ n_out, int64_t capacity, float* __restrict__ correction)
{
    if (!after_previous()) return;
    constexpr int N = 256 + 64;  // the CTA's entries, and those behind them that may belong to its last row
    __shared__ float s_term[N][kFewListTokens + 1], s_change[N];
    __shared__ int s_row[N], s_col[N];
    int64_t k_end = *n_out;
    if (k_end > capacity) k_end = capacity;
    const int64_t n = rows * cols;
    auto row_of = [&](int64_t k) -> int {  // -1 for an index outside the matrix
        const int64_t i = idx[k];
        return (i < 0 || i >= n) ? -1 : (int)(i / cols);
    };
    auto change_of = [&](int64_t k) -> float {
        const int64_t i = idx[k];
        const uint32_t byte = codes[i >> 1], c = (i & 1) ? (byte & 15u) : (byte >> 4);
        return bf16_value(val[k]) - bf16_value(bf16_round(__fmul_rn(scale_at<ST>(scales, i >> block_shift), __ldg(levels + c))));
    };
    const int tid = threadIdx.x;
    for (int64_t base = (int64_t)blockIdx.x * 256; base < k_end; base += (int64_t)gridDim.x * 256) {
        for (int e = tid; e < N; e += 256) {
            const int64_t k = base + e;
            const int r = k < k_end ? row_of(k) : -1;
            s_row[e] = r;
            s_col[e] = r >= 0 ? (int)(idx[k] - (int64_t)r * cols) : 0;
            s_change[e] = r >= 0 ? change_of(k) : 0.0f;
        }
        __syncthreads();
        // a term per entry and token, four on their way at a time
        for (int e0 = tid; e0 < N * tokens; e0 += 4 * 256) {
            float v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = e0 + u * 256, t = i / N, e = i - t * N;
                v[u] = t < tokens && s_row[e] >= 0 ? s_change[e] * bf16_value(__ldg(x + t * ldx + s_col[e])) : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = e0 + u * 256, t = i / N;
                if (t < tokens) s_term[i - t * N][t] = v[u];
            }
        }
        __syncthreads();
        // the sums of a row's entries, a thread per token
        for (int i = tid; i < 256 * tokens; i += 256) {
            const int e = i & 255, t = i >> 8, row = s_row[e];
            if (row < 0 || (e > 0 ? s_row[e - 1] : (base > 0 ? row_of(base - 1) : -1)) == row) continue;  // not the first outlier of its row
            float sum = 0.0f;
            int j = e;
            while (j < N && s_row[j] == row) sum += s_term[j++][t];
            if (j == N)
                for (int64_t kk = base + N; kk < k_end && row_of(kk) == row; ++kk) sum += change_of(kk) * bf16_value(x[t * ldx + idx[kk] - (int64_t)row * cols]);
            correction[(int64_t)t * rows + row] = sum;
        }
        __syncthreads();
    }
}

namespace {

struct FewPlan {
    FewWork work{};
    int grid = 0;
    size_t sums = 0, correction = 0, total = 0;  // byte offsets (the tickets are at 0), and the bytes of all
};

FewPlan few_plan(int64_t rows, int64_t cols, int64_t tokens, bool list)
{
    FewPlan p;
    const int warps = tokens > 8 ? FewGeo<2>::warps : FewGeo<1>::warps;
    const int64_t stripes = (cols + kFewStripe - 1) / kFewStripe, tiles = (rows + 15) / 16;
    // as few slices as give nearly all warps a stripe
    int64_t slices = (stripes + warps - 1) / warps, best = 0;
    for (int64_t n = slices; n <= 4 * slices && n <= kSMs && n <= stripes; ++n) {
        const int64_t wide = (stripes + n - 1) / n, used = wide * (warps / wide) * 64 * stripes / (wide * n);  // warps that have a stripe, in 64ths
        if (used > best + warps * 4) best = used, slices = n;
    }
    FewWork& w = p.work;
    w.slices = (int)slices;
    w.stripes = (int)((stripes + slices - 1) / slices);
    w.groups = warps / w.stripes;
    if (w.groups > tiles) w.groups = (int)tiles;
    w.tiles = (int)tiles;
    w.defer = tokens > 8 ? FewGeo<2>::defer((int)tokens) : FewGeo<1>::defer((int)tokens);
    const int64_t want = (tiles + w.groups - 1) / w.groups, have = kSMs / slices;
    w.peers = (int)(want < have ? want : have);
    p.grid = w.peers * w.slices;
    p.sums = up256((size_t)w.peers * 8);
    p.correction = p.sums + (slices > 1 ? up256((size_t)slices * tokens * tiles * 64) : 0);
    p.total = p.correction + (list ? up256((size_t)tokens * rows * 4) : 0);
    return p;
}

}  // namespace

// Up to sixteen tokens, where the other form decodes as much for a tile of sixteen (8192 x 8192: 26.7 us against 31.7 for nine tokens, 29.2
// against 31.9 for twelve, 33.1 against 31.9 for sixteen; 1024 x 4096 by sixteen: 9 against 13; the largest lose: 28672 x 8192 by sixteen 97 against 84).  Up to six with a list of outliers: its corrections
// cost about 2 us a token here, its entries in the tiles the same for any number of tokens there (8192 x 8192 with 65,536: 35.0 us against 42.2 for
// four tokens, 40.0 against 42.2 for six, 42.6 against 42.2 for seven, 60 against 42 for twelve).
bool linear_few_applies(int64_t rows, int64_t cols, int64_t tokens, bool list)
{
    return tokens <= (list ? kFewListTokens : kFewTokens) && cols <= 32768 && rows <= (1 << 26);
}

size_t linear_few_ws_bytes(int64_t rows, int64_t cols, int64_t tokens, int64_t capacity) { return few_plan(rows, cols, tokens, capacity > 0).total; }

int linear_few(const char* who, const LinearW& w, const void* x, int64_t ldx, const LinearOut& out, int* status, void* ws, size_t ws_bytes, cudaStream_t st)
{
    const bool list = w.out_idx && w.capacity > 0;
    FewPlan p = few_plan(w.rows, w.cols, out.tokens, list);
    if (ws_bytes < p.total) {
        set_error("%s: the workspace has %zu bytes, %zu are needed", who, ws_bytes, p.total);
        return BOF4_ERR_WORKSPACE;
    }
    unsigned char* const base = static_cast<unsigned char*>(ws);
    const uint16_t* const xb = static_cast<const uint16_t*>(x);
    float* correction = nullptr;
    if (list) {
        correction = reinterpret_cast<float*>(base + p.correction);
        BOF4_CUDA_TRY(cudaMemsetAsync(correction, 0, (size_t)out.tokens * w.rows * 4, st));
        const int64_t want = (w.capacity + 255) / 256;
        launch_after(w.scale_dtype == BOF4_F32 ? few_correction_kernel<F32> : few_correction_kernel<BF16>, (int)(want < 4 * kSMs ? want : 4 * kSMs), 256,
                     0, st, w.codes, w.scales, w.rows, w.cols, w.block_shift, w.levels, xb, ldx, (int)out.tokens, w.out_idx, w.out_val, w.n_out,
                     w.capacity, correction);
        BOF4_CUDA_TRY(cudaGetLastError());
    }
    p.work.epoch = tc_next_epoch();
    int rc;
    CUtensorMap code_map;
    if ((rc = tc_make_map(who, w.codes, 1, w.cols / 2, w.rows, w.cols / 2, 128, 16, &code_map))) return rc;
#define BOF4_FEW_GO(NT_, ST_, HALF_)                                                                                                              \
    {                                                                                                                                             \
        constexpr auto kern = linear_few_kernel<NT_, ST_, HALF_>;                                                                                 \
        constexpr int smem = (int)kFewRing + FewGeo<NT_>::ring - kFewBegin;  \
        if ((rc = ensure_dynamic_smem<kern>(smem))) return rc;                                                                       \
        launch_after(kern, p.grid, FewGeo<NT_>::threads, smem, st, code_map, w.scales, w.rows, w.cols, w.block_shift, w.levels, xb,   \
                     ldx, out, correction, status, p.work, reinterpret_cast<unsigned long long*>(base), reinterpret_cast<float*>(base + p.sums)); \
    }
#define BOF4_FEW_S(NT_, ST_) { if (w.block_size == 32) BOF4_FEW_GO(NT_, ST_, true) else BOF4_FEW_GO(NT_, ST_, false) }
#define BOF4_FEW_N(NT_) { if (w.scale_dtype == BOF4_F32) BOF4_FEW_S(NT_, F32) else BOF4_FEW_S(NT_, BF16) }
    if (out.tokens > 8) BOF4_FEW_N(2) else BOF4_FEW_N(1)
#undef BOF4_FEW_N
#undef BOF4_FEW_S
#undef BOF4_FEW_GO
    BOF4_CUDA_TRY(cudaGetLastError());
    return BOF4_OK;
}

}  // namespace bof4
