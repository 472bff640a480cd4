// bof4_cross_entropy: the softmax cross entropy of tokens over a vocabulary whose matrix W is in 4 bits, and the gradient of x.
//
//   z[t, v] = sum_c W^[v, c] x[t, c],   lse[t] = log sum_v exp(z[t, v]),   loss[t] = lse[t] - z[t, y]   (y the token's target)
//   dx[t] = g[t] (sum_v p[t, v] W^[v] - W^[y]),   p = exp(z - lse)
//
// In both forms the target has no part in the sums: with S = sum over v != y of exp(z_v - r) and a = z_y - r for a reference r,
// loss = log(1 + S e^-a) and p_y - 1 = -S / (S + e^a), so that nothing cancels where the target has next to all of the probability.
//
// Few tokens: the logits of all rows (fp32) fit a workspace; the products are those of bof4_linear and its backward pass, which decode as
// they multiply.  Between them one kernel, a CTA per row of up to 16384 logits, or two, for sums of 2048 logits each and for dz.  dz is in bf16, in units
// of g (1 - p_y): the target's entry, often the largest by far, is -1 and needs no rounding, and the second product's results are multiplied by the unit.
//
// Many tokens: the vocabulary in pieces of at most 32768 rows, so that neither logits nor a decoded matrix is kept.  A piece is
// decoded once and multiplied twice (dense_tc.cu): the first product's results become E = exp(z - r) in bf16 and its sums in the
// same kernel, the second adds E W^ to a running sum in fp32, as attention does with its keys as values:
//   dx = g (sum_v E_v W^_v - S W^_y) / (S + e^a)
// That takes two products where recomputing the logits after their sum is known takes three.  r needs no more than to be near the largest
// logit (fp32 and bf16 have room for e^80 either way): it is what the pieces before had, and parts of a piece that lie more than 24 above
// bring their own and are put right before the second product (loss_combine_kernel).  The first piece takes 0 for a guess.
#include "dense_tc.cuh"

namespace bof4 {

constexpr int kCeChunk = 2048;        // logits of a CTA
constexpr int kCePiece = 32768;       // rows of a piece: half as many cost 29 us more per 4096 x 4096 running sums, which are read and written
constexpr int kCePart = 64;           // columns of an entry of the product's sums
constexpr int kCeParts = kCePiece / kCePart;

// What the sums say about a token.
struct CeToken {
    float lse, loss;
    float scale;  // p_v = scale * exp(z_v - r)
    float rest;   // 1 - p_y
};
__device__ __forceinline__ CeToken ce_token(float r, float s, float own, bool counted)
{
    CeToken c;
    if (!counted) {
        c.lse = r + logf(s), c.loss = 0.0f, c.scale = 0.0f, c.rest = 0.0f;
        return c;
    }
    // The others against the target.  Few tokens have r for the largest of the others, so that odds below one mean a > 0; with many tokens r may lie 24 above all of them, and
    // then log(s + e^a) - a would cancel where a < 0 as well.  (Odds of no use, or infinite, where a is far below zero: s is e^-24 at least.)
    const float a = own - r, down = expf(-a), odds = s * down;
    const float none = own - own;  // zero, or NaN where the target's logit is not finite: infinity less infinity, as the loss is
    if (s == 0.0f) {  // nothing but the target
        c.lse = own, c.loss = c.rest = none, c.scale = 0.0f;
    } else if (a > 0.0f || odds <= 1.0f) {
        const float total = 1.0f + odds;
        const float more = log1pf(odds);
        c.loss = more + none, c.lse = own + more, c.scale = down / total, c.rest = odds / total + none;
    } else {
        const float total = s + expf(a);
        c.lse = r + logf(total), c.loss = logf(total) - a, c.scale = 1.0f / total, c.rest = s / total;
    }
    return c;
}
// Two parts' references and sums as one.  A sum of zero has no reference.
__device__ __forceinline__ float2 ce_join(float2 a, float2 b)
{
    if (b.y == 0.0f) return a;
    if (a.y == 0.0f) return b;
    const float r = fmaxf(a.x, b.x);
    return make_float2(r, a.y * __expf(a.x - r) + b.y * __expf(b.x - r));
}
__device__ __forceinline__ float2 ce_join_warp(float2 v)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v = ce_join(v, make_float2(__shfl_xor_sync(kFull, v.x, d), __shfl_xor_sync(kFull, v.y, d)));
    return v;
}

// ---------------------------------------------------------------- few tokens

// Eight logits of a row from column c (those past the end: -inf).
__device__ __forceinline__ void ce_load8(const float* __restrict__ row, int64_t c, int64_t n, float (&v)[8])
{
    if (c + 8 <= n) {
        const float4 a = __ldcg(reinterpret_cast<const float4*>(row + c)), b = __ldcg(reinterpret_cast<const float4*>(row + c) + 1);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = c + k < n ? __ldcg(row + c + k) : -INFINITY;
    }
}
// Reference and sum of a chunk of a token's logits but for the target's, which is kept (13 tokens of 128256: 5.6 us, and 7.7 for the gradients; latency and launches).
__global__ void __launch_bounds__(256)
loss_chunk_kernel(const float* __restrict__ logits, int64_t ld, int64_t n, int chunks, const int64_t* __restrict__ targets, float2* __restrict__ stats,
                  float* __restrict__ own)
{
    if (!after_previous()) return;
    __shared__ float2 s_part[8];
    const int chunk = (int)(blockIdx.x % (unsigned)chunks), tid = threadIdx.x;
    const int64_t t = blockIdx.x / (unsigned)chunks, c = (int64_t)chunk * kCeChunk + tid * 8, target = targets[t];
    float v[8];
    ce_load8(logits + t * ld, c, n, v);
    if (target >= c && target < c + 8 && target < n) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (target == c + k) own[t] = v[k], v[k] = -INFINITY;
    }
    float top = v[0];
#pragma unroll
    for (int k = 1; k < 8; ++k) top = fmaxf(top, v[k]);
    const float r = top > -INFINITY ? top : 0.0f;
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += __expf(v[k] - r);
    const float2 w = ce_join_warp(make_float2(r, sum));
    if ((tid & 31) == 0) s_part[tid >> 5] = w;
    __syncthreads();
    if (tid) return;
    float2 all = s_part[0];
#pragma unroll
    for (int k = 1; k < 8; ++k) all = ce_join(all, s_part[k]);
    stats[t * chunks + chunk] = all;
}

__device__ __forceinline__ bool ce_counted(int64_t target, int64_t n, int* status)
{
    if (target >= n) atomicCAS(status, 0, 2);
    return target >= 0 && target < n;
}
__device__ __forceinline__ float2 ce_join_chunks(const float2* __restrict__ stats, int chunks, int lane)
{
    float2 v = make_float2(0.0f, 0.0f);
    for (int k = lane; k < chunks; k += 32) v = ce_join(v, __ldcg(stats + k));
    return ce_join_warp(v);
}
// Loss and log-sum of each token, a warp each; with gradients, a CTA per chunk of a token's logits: dz.
__global__ void __launch_bounds__(256)
loss_token_kernel(const float2* __restrict__ stats, const float* __restrict__ own, int64_t n, int chunks, const int64_t* __restrict__ targets, int64_t tokens,
                  float* __restrict__ loss, float* __restrict__ lse, int* __restrict__ status)
{
    if (!after_previous()) return;
    const int lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (t >= tokens) return;
    const float2 v = ce_join_chunks(stats + t * chunks, chunks, lane);
    if (lane) return;
    const bool counted = ce_counted(targets[t], n, status);
    const CeToken c = ce_token(v.x, v.y, counted ? own[t] : 0.0f, counted);
    loss[t] = c.loss;
    if (lse) lse[t] = c.lse;
}
__global__ void __launch_bounds__(256)
loss_gradient_kernel(const float* __restrict__ logits, int64_t ld, int64_t n, int chunks, const float2* __restrict__ stats, const float* __restrict__ own,
                     const int64_t* __restrict__ targets, const float* __restrict__ dloss, float* __restrict__ loss, float* __restrict__ lse,
                     float* __restrict__ scale, uint16_t* __restrict__ dz, int* __restrict__ status)
{
    if (!after_previous()) return;
    const int chunk = (int)(blockIdx.x % (unsigned)chunks), tid = threadIdx.x;
    const int64_t t = blockIdx.x / (unsigned)chunks, c0 = (int64_t)chunk * kCeChunk + tid * 8, target = targets[t];
    float v[8];
    if (c0 < n) ce_load8(logits + t * ld, c0, n, v);  // on their way meanwhile
    const float2 s = ce_join_chunks(stats + t * chunks, chunks, tid & 31);
    const bool counted = target >= 0 && target < n;
    const CeToken c = ce_token(s.x, s.y, counted ? own[t] : 0.0f, counted);
    if (chunk == 0 && tid == 0) {
        ce_counted(target, n, status);
        loss[t] = c.loss;
        if (lse) lse[t] = c.lse;
        scale[t] = counted ? (dloss ? dloss[t] : 1.0f) * c.rest : 0.0f;
    }
    if (c0 >= n) return;
    const float unit = 1.0f / s.y;  // p_v / (1 - p_y) = exp(z_v - r) / S
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = !counted || s.y == 0.0f ? 0.0f : target == c0 + k ? -1.0f : unit * __expf(v[k] - s.x);
    // (rows are padded to eight)
    *reinterpret_cast<uint4*>(dz + t * ld + c0) = make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
}

// All of this for a token whose logits one CTA can keep in its registers: loss, log-sum, and dz where it is wanted.
constexpr int kCeRow = 16384;  // 1024 threads, twice eight logits each (one token of 32000 in one CTA took 1 us longer than in chunks)
template <bool GRAD>
__global__ void __launch_bounds__(1024)
loss_row_kernel(const float* __restrict__ logits, int64_t ld, int n, const int64_t* __restrict__ targets, const float* __restrict__ dloss, float* __restrict__ loss,
                float* __restrict__ lse, float* __restrict__ scale, uint16_t* __restrict__ dz, int* __restrict__ status)
{
    if (!after_previous()) return;
    __shared__ float s_top[32], s_sum[32], s_own;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t t = blockIdx.x, target = targets[t];
    const float* const row = logits + t * ld;
    constexpr int N = kCeRow / 8192;
    float v[N][8], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if ((tid + i * 1024) * 8 < n) ce_load8(row, (tid + i * 1024) * 8, n, v[i]);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = (tid + i * 1024) * 8;
        if (c >= n) break;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (target == c + k && c + k < n) s_own = v[i][k], v[i][k] = -INFINITY;
            top = fmaxf(top, v[i][k]);
        }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, d));
    if (lane == 0) s_top[warp] = top;
    __syncthreads();
    top = s_top[lane];
#pragma unroll
    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, d));
    const float r = top > -INFINITY ? top : 0.0f;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if ((tid + i * 1024) * 8 >= n) break;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            v[i][k] = __expf(v[i][k] - r);
            sum += v[i][k];
        }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(kFull, sum, d);
    if (lane == 0) s_sum[warp] = sum;
    __syncthreads();
    sum = s_sum[lane];
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(kFull, sum, d);
    const bool counted = target >= 0 && target < n;
    if (tid == 0) {
        ce_counted(target, n, status);
        const CeToken c = ce_token(r, sum, counted ? s_own : 0.0f, counted);
        loss[t] = c.loss;
        if (lse) lse[t] = c.lse;
        if (GRAD) scale[t] = counted ? (dloss ? dloss[t] : 1.0f) * c.rest : 0.0f;
    }
    if (!GRAD) return;
    const float unit = 1.0f / sum;  // p_v / (1 - p_y) = exp(z_v - r) / S
    const bool any = counted && sum != 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = (tid + i * 1024) * 8;
        if (c >= n) break;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[i][k] = !any ? 0.0f : target == c + k ? -1.0f : unit * v[i][k];
        *reinterpret_cast<uint4*>(dz + t * ld + c) =
            make_uint4(bf16_pair(v[i][0], v[i][1]), bf16_pair(v[i][2], v[i][3]), bf16_pair(v[i][4], v[i][5]), bf16_pair(v[i][6], v[i][7]));
    }
}

// ---------------------------------------------------------------- many tokens

// A piece's sums joined with those of the pieces before; E of parts that used another reference is put right.  32 tokens a CTA, a warp every 32nd part of the
// piece, kept in registers (4096 tokens, 512 parts: 9 us, latency).
__global__ void __launch_bounds__(1024)
loss_combine_kernel(const float2* __restrict__ stats, int parts, int64_t tokens, bool first, float* __restrict__ ref, float* __restrict__ sum,
                    float* __restrict__ factor, uint16_t* __restrict__ e, int64_t ld, int64_t n)
{
    if (!after_previous()) return;
    __shared__ float2 s_part[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t t = (int64_t)blockIdx.x * 32 + lane;
    const bool live = t < tokens;
    constexpr int N = kCeParts / 32;
    float2 v[N], all = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = live && warp + 32 * k < parts ? __ldcg(stats + (int64_t)(warp + 32 * k) * tokens + t) : make_float2(0.0f, 0.0f);
#pragma unroll
    for (int k = 0; k < N; ++k) all = ce_join(all, v[k]);
    s_part[warp][lane] = all;
    __syncthreads();
    // a warp joins the 32 warps' parts of one token
    const int64_t mine = (int64_t)blockIdx.x * 32 + warp;
    const float2 w = ce_join_warp(s_part[lane][warp]);
    float2 old = make_float2(0.0f, 0.0f);
    if (mine < tokens && !first) old = make_float2(ref[mine], sum[mine]);
    const float2 now = ce_join(old, w);
    __syncthreads();
    if (lane == 0) {
        s_part[0][warp] = now;
        if (mine < tokens) {
            ref[mine] = now.y == 0.0f ? -INFINITY : now.x, sum[mine] = now.y;  // (no reference yet: the next piece's parts bring theirs)
            factor[mine] = old.y == 0.0f ? 0.0f : __expf(old.x - now.x);
        }
    }
    __syncthreads();
    if (!e) return;
    const float to = s_part[0][lane].x;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const float f = v[k].y == 0.0f ? 1.0f : __expf(v[k].x - to);
        unsigned int rows = __ballot_sync(kFull, v[k].y != 0.0f && v[k].x != to);
        while (rows) {
            const int j = __ffs((int)rows) - 1;
            rows &= rows - 1;
            const float fj = __shfl_sync(kFull, f, j);
            const int64_t c = (int64_t)(warp + 32 * k) * kCePart + 2 * lane;
            if (c >= n) continue;
            uint32_t* const p = reinterpret_cast<uint32_t*>(e + ((int64_t)blockIdx.x * 32 + j) * ld + c);  // (rows are padded to eight)
            const uint32_t u = *p;
            *p = bf16_pair(__uint_as_float(u << 16) * fj, __uint_as_float(u & 0xffff0000u) * fj);
        }
    }
}

// Outliers of the rows of a piece over its decoded weights.
__global__ void __launch_bounds__(256)
loss_outliers_kernel(const int32_t* __restrict__ idx, const uint16_t* __restrict__ val, const int64_t* __restrict__ n_out, int64_t capacity, int64_t begin,
                     int64_t count, uint16_t* __restrict__ w)
{
    if (!after_previous()) return;
    const int64_t end = *n_out < capacity ? *n_out : capacity;
    for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < end; k += (int64_t)gridDim.x * 256) {
        const int64_t i = idx[k] - begin;
        if (i >= 0 && i < count) w[i] = val[k];
    }
}

struct LossFinal {
    const float *ref, *sum, *own, *acc, *dloss;
    const int64_t* targets;
    int64_t rows, cols, tokens;
    float *loss, *lse;
    uint16_t* dx;
    int64_t ld_dx;
    bool wide;  // rows of dx begin at multiples of 16 bytes
    int* status;
    const uint8_t* codes;
    const void* scales;
    const float* levels;
    int block_shift;
    const int32_t* idx;  // NULL without a list
    const uint16_t* val;
    const int64_t* n_out;
    int64_t capacity;
};
__global__ void __launch_bounds__(256) loss_value_kernel(const LossFinal f)
{
    if (!after_previous()) return;
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t >= f.tokens) return;
    const bool counted = ce_counted(f.targets[t], f.rows, f.status);
    const CeToken c = ce_token(f.ref[t], f.sum[t], counted ? f.own[t] : 0.0f, counted);
    f.loss[t] = c.loss;
    if (f.lse) f.lse[t] = c.lse;
}
// dx of a token, a CTA each: the running sum less the target's row, which is decoded here (4096 tokens of 4096 columns 18 us, 110 MB).
template <class ST>
__global__ void __launch_bounds__(256) loss_dx_kernel(const LossFinal f)
{
    if (!after_previous()) return;
    __shared__ float s_levels[16];
    const int64_t t = blockIdx.x, target = f.targets[t];
    const int tid = threadIdx.x;
    if (tid < 16) s_levels[tid] = __ldg(f.levels + tid);
    const bool counted = target >= 0 && target < f.rows;
    const CeToken c = ce_token(f.ref[t], f.sum[t], counted ? f.own[t] : 0.0f, counted);
    if (tid == 0) {
        ce_counted(target, f.rows, f.status);
        f.loss[t] = c.loss;
        if (f.lse) f.lse[t] = c.lse;
    }
    __syncthreads();
    const float g = f.dloss ? f.dloss[t] : 1.0f;
    uint16_t* const dx = f.dx + t * f.ld_dx;
    const float* const acc = f.acc + t * f.cols;
    const int64_t first = target * f.cols;
    for (int64_t o = tid * 8; o < f.cols; o += 256 * 8) {  // (eight columns are in one block)
        float v[8];
        if (!counted) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = 0.0f;
        } else {
            const uint32_t code = *reinterpret_cast<const uint32_t*>(f.codes + ((first + o) >> 1));
            const int64_t b = (first + o) >> f.block_shift;
            const float m = ST::code == BOF4_F32 ? __ldg(static_cast<const float*>(f.scales) + b) : bf16_value(__ldg(static_cast<const uint16_t*>(f.scales) + b));
            const float4 a0 = *reinterpret_cast<const float4*>(acc + o), a1 = *reinterpret_cast<const float4*>(acc + o + 4);
            const float a[8] = {a0.x, a0.y, a0.z, a0.w, a1.x, a1.y, a1.z, a1.w};
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t byte = code >> (k >> 1) * 8;
                const float w = bf16_value(bf16_round(__fmul_rn(m, s_levels[k & 1 ? byte & 15u : byte >> 4 & 15u])));
                v[k] = g * (c.scale * a[k] - c.rest * w);
            }
        }
        if (f.wide) {
            *reinterpret_cast<uint4*>(dx + o) = make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) dx[o + k] = bf16_round(v[k]);
        }
    }
    if (!f.idx || !counted) return;
    // columns of the target's row that hold an outlier, once more
    int64_t end = *f.n_out < f.capacity ? *f.n_out : f.capacity, lo = 0, hi = end;
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (f.idx[mid] < first) lo = mid + 1;
        else hi = mid;
    }
    __syncthreads();
    for (int64_t k = lo + tid; k < end; k += 256) {
        const int64_t o = f.idx[k] - first;
        if (o >= f.cols) break;
        dx[o] = bf16_round(g * (c.scale * acc[o] - c.rest * bf16_value(f.val[k])));
    }
}

// ---------------------------------------------------------------- host side

namespace {

// Whether the vocabulary is taken in pieces.  Both forms, us, decoding as it multiplies against this: with the gradient 16000 x 4096 by 256 125 against 123, 32000 x 4096 by 257
// 278 against 274, 512 379 against 285, 128256 x 4096 by 257 1046 against 1083, 384 1331 against 1165, 128256 x 8192 by 257 2242 against 1926; without it 32000 x 4096 by 384
// 173 against 182, 448 194 against 195, 512 239 against 178, 50000 x 4096 by 384 243 against 249, 448 270 against 251, 128256 x 4096 by 385 589 against 643, 448 668 against 655.
// With few columns sooner: 60000 x 512 by 130 without the gradient 83 against 62, with it by 200 198 against 171; x 1088 by 130 93 against 83, with it by 200 209 against 204; x 2048 by
// 200 134 against 132, with it by 256 270 against 255.
bool loss_dense(int64_t cols, int64_t tokens, bool grad)
{
    return tokens > (cols <= 1088 && !grad ? 128 : cols <= 2048 ? 192 : grad ? 256 : 384);
}

struct LossPlan {
    bool dense;
    int64_t ld;                  // of logits, of E
    int chunks;                  // few tokens
    int64_t pieces, piece;       // many
    size_t forward, backward;    // bytes of the products' workspaces, which share a place
    size_t logits, stats, own, scale, dz, w, ref, sum, factor, acc, total;
};
bool loss_plan(int64_t rows, int64_t cols, int64_t tokens, bool grad, int64_t capacity, LossPlan* p)
{
    p->dense = loss_dense(cols, tokens, grad);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += up256(bytes);
        return here;
    };
    const size_t t = (size_t)tokens;
    if (!p->dense) {
        p->forward = few_pays(rows, cols, tokens, capacity > 0) ? linear_few_ws_bytes(rows, cols, tokens, capacity, true)
                                                                          : linear_tc_ws_bytes(rows, cols, tokens, false, capacity);
        p->backward = grad ? linear_tc_ws_bytes(rows, cols, tokens, true, capacity) : 0;
        if (!p->forward || (grad && !p->backward)) return false;
        at = up256(p->forward > p->backward ? p->forward : p->backward);
        p->ld = (rows + 7) & ~(int64_t)7;
        const int64_t chunks = (rows + kCeChunk - 1) / kCeChunk;
        if (chunks * tokens > INT32_MAX) return false;
        p->chunks = (int)chunks;
        p->logits = take(t * p->ld * 4);
        p->stats = take(t * chunks * 8);
        p->own = take(t * 4);
        p->scale = take(t * 4);
        p->dz = take(grad ? t * p->ld * 2 : 0);
        p->total = at;
        return true;
    }
    p->pieces = (rows + kCePiece - 1) / kCePiece;
    p->piece = ((rows + p->pieces - 1) / p->pieces + 255) & ~(int64_t)255;
    p->ld = p->piece;
    p->forward = p->backward = dense_ws_most();
    if (!dense_ws_bytes(tokens, p->piece, cols) || !dense_ws_bytes(tokens, cols, p->piece)) return false;
    at = up256(p->forward);
    p->w = take((size_t)p->piece * cols * 2);
    p->stats = take(t * kCeParts * 8);
    p->own = take(t * 4);
    p->ref = take(t * 4);
    p->sum = take(t * 4);
    p->factor = take(t * 4);
    p->dz = take(grad ? t * p->ld * 2 : 0);
    p->acc = take(grad ? t * cols * 4 : 0);
    p->total = at;
    return true;
}

}  // namespace
}  // namespace bof4

using namespace bof4;

extern "C" size_t bof4_cross_entropy_workspace_bytes(int64_t rows, int64_t cols, int64_t n_tokens, int want_dx, int64_t capacity)
{
    if (rows < 0 || cols < 0 || n_tokens < 0 || capacity < 0 || rows > INT32_MAX || cols > INT32_MAX || n_tokens > INT32_MAX || capacity > INT32_MAX)
        return 0;
    if (n_tokens == 0) return 256;
    LossPlan p;
    return rows && cols && loss_plan(rows, cols, n_tokens, want_dx != 0, capacity, &p) ? p.total : 0;
}

extern "C" int bof4_cross_entropy(const uint8_t* d_codes, const void* d_scales, int scale_dtype, int64_t rows, int64_t cols, int block_size,
                                  const float* d_codebook, const void* d_x, int64_t ldx, int64_t n_tokens, const int64_t* d_targets,
                                  const float* d_dloss, const int32_t* d_out_idx, const void* d_out_val, const int64_t* d_n_out, int64_t capacity,
                                  float* d_loss, float* d_lse, void* d_dx, int64_t ld_dx, int* d_status, void* d_ws, size_t ws_bytes, void* stream)
{
    const char* fn = "bof4_cross_entropy";
    LinearW w{};
    if (const int rc = linear_check(fn, &w, d_scales, scale_dtype, rows, cols, block_size, n_tokens, BOF4_ACT_NONE, d_out_idx, d_out_val, d_n_out, capacity))
        return rc;
    if (n_tokens > 0 && (rows == 0 || cols == 0)) {
        set_error("%s: a vocabulary without rows or columns", fn);
        return BOF4_ERR_SHAPE;
    }
    if (n_tokens > 1 && (ldx < cols || (d_dx && ld_dx < cols))) {
        set_error("%s: a row stride is smaller than its row", fn);
        return BOF4_ERR_SHAPE;
    }
    if (!d_status) {
        set_error("%s: NULL status pointer", fn);
        return BOF4_ERR_INVALID_ARG;
    }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (n_tokens == 0) {
        BOF4_CUDA_TRY(cudaMemsetAsync(d_status, 0, sizeof(int), st));
        return BOF4_OK;
    }
    if (!d_codes || !d_scales || !d_codebook || !d_x || !d_targets || !d_loss) {
        set_error("%s: NULL pointer", fn);
        return BOF4_ERR_INVALID_ARG;
    }
    if (n_tokens == 1) ldx = cols, ld_dx = cols;
    if (!aligned32(d_codes) || !aligned16(d_x) || ldx % 8) {
        set_error("%s: d_codes must be 32-byte aligned, d_x 16-byte aligned and ldx a multiple of 8", fn);
        return BOF4_ERR_INVALID_ARG;
    }
    const bool grad = d_dx != nullptr;
    LossPlan p;
    if (!loss_plan(rows, cols, n_tokens, grad, w.capacity, &p)) {
        set_error("%s: matrix or batch too large", fn);
        return BOF4_ERR_SHAPE;
    }
    if (!d_ws || (reinterpret_cast<uintptr_t>(d_ws) & 255u) || ws_bytes < p.total) {
        set_error("%s: the workspace must be 256-byte aligned and hold %zu bytes", fn, p.total);
        return BOF4_ERR_WORKSPACE;
    }
    w.codes = d_codes;
    w.levels = d_codebook;
    unsigned char* const base = static_cast<unsigned char*>(d_ws);
    auto floats = [&](size_t at) { return reinterpret_cast<float*>(base + at); };
    float2* const stats = reinterpret_cast<float2*>(base + p.stats);
    float* const own = floats(p.own);
    uint16_t* const dz = reinterpret_cast<uint16_t*>(base + p.dz);
    int rc;
    if (!p.dense) {
        float* const logits = floats(p.logits);
        LinearOut out{};
        out.y = logits;
        out.ldy = p.ld;
        out.n = rows;
        out.tokens = n_tokens;
        out.few_parts = true;
        out.set_alignment();
        if (few_pays(rows, cols, n_tokens, w.capacity > 0)) rc = linear_few(fn, w, d_x, ldx, out, d_status, base, p.forward, st);
        else rc = linear_tc(fn, w, false, d_x, ldx, out, d_status, base, p.forward, st);
        if (rc) return rc;
        float* const scale = floats(p.scale);
        if (rows <= kCeRow) {
            if (grad) launch_after(loss_row_kernel<true>, (int)n_tokens, 1024, 0, st, logits, p.ld, (int)rows, d_targets, d_dloss, d_loss, d_lse, scale, dz, d_status);
            else launch_after(loss_row_kernel<false>, (int)n_tokens, 1024, 0, st, logits, p.ld, (int)rows, d_targets, nullptr, d_loss, d_lse, nullptr, nullptr, d_status);
        } else {
            launch_after(loss_chunk_kernel, (int)(p.chunks * n_tokens), 256, 0, st, logits, p.ld, rows, p.chunks, d_targets, stats, own);
            if (grad)
                launch_after(loss_gradient_kernel, (int)(p.chunks * n_tokens), 256, 0, st, logits, p.ld, rows, p.chunks, stats, own, d_targets, d_dloss, d_loss,
                             d_lse, scale, dz, d_status);
            else
                launch_after(loss_token_kernel, (int)((n_tokens + 7) / 8), 256, 0, st, stats, own, rows, p.chunks, d_targets, n_tokens, d_loss, d_lse, d_status);
        }
        BOF4_CUDA_TRY(cudaGetLastError());
        if (!grad) return BOF4_OK;
        LinearOut to{};
        to.y = d_dx;
        to.ldy = ld_dx;
        to.y_bf16 = true;
        to.n = cols;
        to.tokens = n_tokens;
        to.keep_status = true;
        to.scale = scale;
        to.few_parts = true;
        to.set_alignment();
        return linear_tc(fn, w, true, dz, p.ld, to, d_status, base, p.backward, st);
    }
    float *const ref = floats(p.ref), *const sum = floats(p.sum), *const factor = floats(p.factor), *const acc = floats(p.acc);
    void* const decoded = base + p.w;
    for (int64_t r0 = 0; r0 < rows; r0 += p.piece) {
        const int64_t n = rows - r0 < p.piece ? rows - r0 : p.piece;
        const bool first = r0 == 0;
        const size_t scale_bytes = scale_dtype == BOF4_F32 ? 4 : 2;
        if ((rc = bof4_dequantize(d_codes + r0 * cols / 2, static_cast<const unsigned char*>(d_scales) + (size_t)(r0 * cols / block_size) * scale_bytes, scale_dtype,
                                  n * cols, block_size, d_codebook, nullptr, nullptr, nullptr, 0, decoded, BOF4_BF16, st)))
            return rc;
        if (w.capacity) {
            const int64_t want = (w.capacity + 255) / 256;
            launch_after(loss_outliers_kernel, (int)(want < 4 * kSMs ? want : 4 * kSMs), 256, 0, st, w.out_idx, w.out_val, w.n_out, w.capacity, r0 * cols, n * cols,
                         static_cast<uint16_t*>(decoded));
        }
        DenseOut out{};
        out.tokens = n_tokens;
        out.n = n;
        out.y = grad ? dz : nullptr;
        out.ldy = p.ld;
        out.targets = d_targets;
        out.first_row = r0;
        out.ref = ref;
        out.stats = stats;
        out.target_logit = own;
        out.first = first;
        out.keep_status = !first;
        if ((rc = dense_product(fn, DenseProduct{d_x, ldx, decoded, 0, cols, n, false, kDenseLoss}, out, d_status, base, p.forward, st))) return rc;
        launch_after(loss_combine_kernel, (int)((n_tokens + 31) / 32), 1024, 0, st, stats, (int)((n + kCePart - 1) / kCePart), n_tokens, first, ref, sum, factor,
                     grad ? dz : nullptr, p.ld, n);
        BOF4_CUDA_TRY(cudaGetLastError());
        if (!grad) continue;
        DenseOut to{};
        to.tokens = n_tokens;
        to.n = cols;
        to.y = acc;
        to.ldy = cols;
        to.factor = first ? nullptr : factor;
        to.keep_status = true;
        if ((rc = dense_product(fn, DenseProduct{dz, p.ld, decoded, 0, n, cols, true, kDenseAdd}, to, d_status, base, p.forward, st))) return rc;
    }
    LossFinal f{};
    f.ref = ref;
    f.sum = sum;
    f.own = own;
    f.acc = acc;
    f.dloss = d_dloss;
    f.targets = d_targets;
    f.rows = rows;
    f.cols = cols;
    f.tokens = n_tokens;
    f.loss = d_loss;
    f.lse = d_lse;
    f.dx = static_cast<uint16_t*>(d_dx);
    f.ld_dx = ld_dx;
    f.wide = aligned16(d_dx) && ld_dx % 8 == 0;
    f.status = d_status;
    f.codes = d_codes;
    f.scales = d_scales;
    f.levels = d_codebook;
    f.block_shift = w.block_shift;
    f.idx = w.capacity ? w.out_idx : nullptr;
    f.val = w.out_val;
    f.n_out = w.n_out;
    f.capacity = w.capacity;
    if (!grad) launch_after(loss_value_kernel, (int)((n_tokens + 255) / 256), 256, 0, st, f);
    else launch_after(scale_dtype == BOF4_F32 ? loss_dx_kernel<F32> : loss_dx_kernel<BF16>, (int)n_tokens, 256, 0, st, f);
    BOF4_CUDA_TRY(cudaGetLastError());
    return BOF4_OK;
}
