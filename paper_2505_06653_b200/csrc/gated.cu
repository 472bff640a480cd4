// Entry points of bof4_gated and bof4_gated_backward: both projections of a gated block, its activation and their product, and the
// gradient of x.  With z = x W^T (+ bias), W of 2 F rows (gate, then up):
//
//   forward   h[t, f] = act(z[t, f]) z[t, F + f]
//   backward  dz[t, f] = dh[t, f] z[t, F + f] act'(z[t, f]),   dz[t, F + f] = dh[t, f] act(z[t, f]),   dx = dz W
//
// The products are those of bof4_linear with gate and up rows in turn, so that a tile has both sums of a column of h: the form
// for few tokens (linear_few.cu), the one that decodes as it multiplies (linear_tc.cuh), and, for many tokens, a decoded matrix and
// a product of plain operands (dense_tc.cu).  z itself is written where a backward pass will want it and never read here.
// The backward product is that of bof4_linear_backward over all 2 F rows at once.
#include <type_traits>

#include "dense_tc.cuh"

namespace bof4 {

// d, gate, up of eight elements -> the two gradients in the places of gate and up; one branch for all of them.
__device__ __forceinline__ void activate_gradients(const float (&d)[8], float (&g)[8], float (&up)[8], int act)
{
    auto all = [&](int which) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float v, slope;
            activate_both(g[k], which, v, slope);
            g[k] = d[k] * up[k] * slope, up[k] = d[k] * v;
        }
    };
    switch (act) {
        case BOF4_ACT_RELU: all(BOF4_ACT_RELU); break;
        case BOF4_ACT_GELU: all(BOF4_ACT_GELU); break;
        case BOF4_ACT_GELU_TANH: all(BOF4_ACT_GELU_TANH); break;
        case BOF4_ACT_SILU: all(BOF4_ACT_SILU); break;
        default: all(BOF4_ACT_NONE);
    }
}

// dz of a gated block, rounded to bf16 for the tensor cores, and the sums of the unrounded dz over a CTA's tokens: as dz_kernel
// (linear.cu), with two results per element.  Sums are added in a fixed order.  One pass over dh and pre, bound by memory: 4096 tokens of 14336 columns by SILU 91 us,
// 587 MB at 6.45 TB/s (170 us with four tokens a warp on their way: 113 registers left two CTAs an SM).
// VEC: a lane has eight neighbouring columns, in one load; where rows begin at odd places or end inside of eight, every 32nd column, so that the lanes of
// a load are neighbours (a whole backward pass of 2653 tokens, 22957 columns by GELU with the bias gradient and K = 640: 682 us with eight neighbours a lane, 411 this way).
template <class DT>
struct DzLoads {  // of the lane's eight columns, as they are in memory
    typename std::conditional<DT::code == BOF4_F32, float, uint16_t>::type v[8];
    __device__ __forceinline__ void load(const void* p, int64_t at, int count)
    {
        using T = typename std::conditional<DT::code == BOF4_F32, float, uint16_t>::type;
        const T* const q = static_cast<const T*>(p) + at;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = 32 * k < count ? __ldg(q + 32 * k) : T(0);
    }
    __device__ __forceinline__ void values(float (&f)[8]) const
    {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if constexpr (DT::code == BOF4_F32) f[k] = v[k];
            else f[k] = bf16_value(v[k]);
        }
    }
};
template <class DT, bool SUMS, bool VEC>
__global__ void __launch_bounds__(256, SUMS ? 2 : DT::code == BOF4_F32 || !VEC ? 3 : 4)
gated_dz_kernel(const void* __restrict__ dh, int64_t ld_dh, const uint16_t* __restrict__ pre, int64_t ld_pre, int act, int64_t n, int64_t tokens,
                uint16_t* __restrict__ dz, int64_t ld_dz, float* __restrict__ sums, int col_blocks, int per)
{
    if (!after_previous()) return;
    __shared__ float s_sum[SUMS ? 8 : 1][2 * kDzCols + 4];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int kLane = VEC ? 8 : 1, kNext = VEC ? 1 : 32;  // between the columns of two lanes, of a lane
    const int64_t chunk = blockIdx.x / col_blocks, c0 = (int64_t)(blockIdx.x % col_blocks) * kDzCols + lane * kLane;
    const int count = (int)(n - c0 < kDzCols ? n - c0 : kDzCols);  // columns from the lane's first
    float sum[16] = {};
    if (count > 0) {
        constexpr int N = 2;  // tokens on their way at a time: more cost warps
#pragma unroll 1
        for (int64_t t0 = chunk * per + warp; t0 < chunk * per + per && t0 < tokens; t0 += 8 * N) {
            typename std::conditional<VEC, Dz8<DT>, DzLoads<DT>>::type a[N];
            typename std::conditional<VEC, Dz8<BF16>, DzLoads<BF16>>::type b[N], c[N];
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int64_t t = t0 + 8 * u;
                if (t >= tokens || t >= chunk * per + per) break;
                if constexpr (VEC) {
                    a[u].load(dh, t * ld_dh + c0, 8, true);
                    b[u].load(pre, t * ld_pre + c0, 8, true);
                    c[u].load(pre, t * ld_pre + n + c0, 8, true);
                } else {
                    a[u].load(dh, t * ld_dh + c0, count);
                    b[u].load(pre, t * ld_pre + c0, count);
                    c[u].load(pre, t * ld_pre + n + c0, count);
                }
            }
#pragma unroll
            for (int u = 0; u < N; ++u) {
                if (t0 + 8 * u >= tokens || t0 + 8 * u >= chunk * per + per) break;
                float d[8], g[8], up[8];
                a[u].values(d);
                b[u].values(g);
                c[u].values(up);
                activate_gradients(d, g, up, act);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (SUMS && (VEC || 32 * k < count)) sum[k] += g[k], sum[8 + k] += up[k];
                if (!dz) continue;
                uint16_t* const p = dz + (t0 + 8 * u) * ld_dz + c0;
                if (VEC) {
                    *reinterpret_cast<uint4*>(p) = make_uint4(bf16_pair(g[0], g[1]), bf16_pair(g[2], g[3]), bf16_pair(g[4], g[5]), bf16_pair(g[6], g[7]));
                    *reinterpret_cast<uint4*>(p + n) = make_uint4(bf16_pair(up[0], up[1]), bf16_pair(up[2], up[3]), bf16_pair(up[4], up[5]), bf16_pair(up[6], up[7]));
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (32 * k < count) p[32 * k] = bf16_round(g[k]), p[n + 32 * k] = bf16_round(up[k]);
                }
            }
        }
    }
    if constexpr (SUMS) {
#pragma unroll
        for (int k = 0; k < 8; ++k) s_sum[warp][lane * kLane + k * kNext] = sum[k], s_sum[warp][kDzCols + lane * kLane + k * kNext] = sum[8 + k];
        __syncthreads();
        const int64_t c = (int64_t)(blockIdx.x % col_blocks) * kDzCols + threadIdx.x;
        if (c < n) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float s = 0.0f;
#pragma unroll
                for (int w = 0; w < 8; ++w) s += s_sum[w][h * kDzCols + threadIdx.x];
                sums[chunk * 2 * n + h * n + c] = s;
            }
        }
    }
}

// The result where there is nothing to multiply (no columns).
__global__ void __launch_bounds__(256) gated_empty_kernel(const LinearOut out, int* __restrict__ status)
{
    if (!after_previous()) return;
    if (blockIdx.x == 0 && threadIdx.x == 0) *status = 0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < out.tokens * out.n; i += (int64_t)gridDim.x * 256)
        out.store_pair(0.0f, 0.0f, i / out.n, i % out.n);
}

namespace {

// Whether a matrix is decoded once and multiplied as plain bf16.  Both forms, us, ffn x columns by tokens, decoding as it multiplies against this:
//   forward    2048 x 2048 by 257 28 against 28, 512 34 against 28; 4096 x 2048 by 512 39 against 32; 8192 x 4096 by 512 80 against 85, 768 105 against 103;
//              11008 x 4096 by 512 104 against 118, 768 139 against 140, 1024 185 against 167; 28672 x 8192 by 896 768 against 814, 1024 841 against 827;
//              with few columns its results take longer than its products: 24184 x 832 (z kept) by 200 72 against 55, 450 147 against 82, x 2048 by 256 98 against 104, 300
//              139 against 131, 600 243 against 156, x 2560 by 300 152 against 160, 450 195 against 165; 8000 x 1088 by 200 27 against 27, 256 29 against 27
//   backward   2048 x 2048 by 448 42 against 40; 4096 x 4096 by 512 63 against 60; 8192 x 4096 by 768 118 against 128; 11008 x 4096 by 768 165 against 175,
//              1024 218 against 194; 28672 x 8192, where the parts of a tile are many, by 384 509 against 544, 448 561 against 560, 512 621 against 556, 1024 1328 against 902
//   between and beside them, in a graph on one box: backward 14336 x 4096 by 640 174 against 204, 768 193 against 208, 896 265 against 224, 14336 x 8192 by 448 255 against 274, 640 367
//              against 345, 896 527 against 456; forward 14336 x 4096 by 512 143 against 157, 640 191 against 174, 28672 x 8192 by 768 613 against 697, 896 777 against 812.  So the one
//              limit of the forward form costs 9 % at the first of these two shapes and 13 % at the second, next to it, the backward limits 6 % at 14336 x 8192
//   h in fp32  whose sums have an accumulator per 1024 of K (linear_tc.cuh): 22016 x 4096 by 257 94 against 110, 384 108 against 112, 512 131 against 112, 767 194 against 135; 57344 x 8192 by
//              384 511 against 520, 512 672 against 536; 11264 x 2048 by 512 53 against 40
bool gated_dense(int64_t rows, int64_t cols, int64_t tokens, bool backward, bool fp32)
{
    const int64_t n = rows * cols;
    if (backward) return tokens >= (n <= (int64_t)1 << 25 || n >= (int64_t)1 << 28 ? 448 : 896);
    return tokens >= 768 || (tokens > 384 && (cols <= 2560 || fp32)) || (tokens > 256 && (cols <= 2048 || n <= (int64_t)1 << 24)) || (tokens > 160 && cols <= 1088);
}

// Parts of the workspace behind the product's: the decoded matrix, dz, the sums of dz.  (cols = 0: no product, and dz is not kept.)
struct GatedPlan {
    bool dense;
    int per;  // tokens of a CTA that forms dz: fewer where there would be less than four CTAs an SM (131 tokens of 11008: 15 us with 32)
    int64_t chunks, ld;
    size_t product, w, dz, sums, total;
};
// False: too large.
bool gated_plan(int64_t ffn, int64_t cols, int64_t tokens, bool backward, bool fp32, int64_t capacity, GatedPlan* p)
{
    const int64_t rows = 2 * ffn;
    p->dense = gated_dense(rows, cols, tokens, backward, fp32);
    p->product = 256;
    if (cols) {
        if (p->dense) p->product = backward ? dense_ws_bytes(tokens, cols, rows) : dense_ws_bytes(tokens, rows, cols);
        else if (!backward && few_pays(rows, cols, tokens, capacity > 0)) p->product = linear_few_ws_bytes(rows, cols, tokens, capacity, true);
        else p->product = linear_tc_ws_bytes(rows, cols, tokens, backward, capacity);
        if (!p->product) return false;
    }
    const int64_t blocks = (ffn + kDzCols - 1) / kDzCols;
    p->per = kDzTokens;
    while (p->per > 8 && (tokens + p->per - 1) / p->per * blocks < 4 * kSMs) p->per /= 2;
    p->chunks = (tokens + p->per - 1) / p->per;
    p->ld = (rows + 7) & ~(int64_t)7;
    p->w = up256(p->product);
    p->dz = p->w + (p->dense ? up256((size_t)rows * cols * 2) : 0);
    p->sums = p->dz + (backward && cols ? up256((size_t)tokens * p->ld * 2) : 0);
    p->total = p->sums + (backward && p->chunks > 1 ? up256((size_t)p->chunks * rows * 4) : 0);
    return true;
}

int gated_decode(const LinearW& w, void* to, cudaStream_t st)
{
    return bof4_dequantize(w.codes, w.scales, w.scale_dtype, w.rows * w.cols, w.block_size, w.levels, w.out_idx, w.out_val, w.n_out, w.capacity, to,
                           BOF4_BF16, st);
}

}  // namespace
}  // namespace bof4

using namespace bof4;

extern "C" size_t bof4_gated_workspace_bytes(int64_t ffn, int64_t cols, int64_t n_tokens, int backward, int64_t capacity)
{
    if (ffn < 0 || cols < 0 || n_tokens < 0 || capacity < 0 || ffn > INT32_MAX / 2 || cols > INT32_MAX || n_tokens > INT32_MAX || capacity > INT32_MAX)
        return 0;
    if (ffn == 0 || n_tokens == 0) return 256;
    GatedPlan p, q;  // for results in bf16 and in fp32
    if (!gated_plan(ffn, cols, n_tokens, backward != 0, false, capacity, &p) || !gated_plan(ffn, cols, n_tokens, backward != 0, true, capacity, &q)) return 0;
    return p.total > q.total ? p.total : q.total;
}

extern "C" int bof4_gated(const uint8_t* d_codes, const void* d_scales, int scale_dtype, int64_t ffn, int64_t cols, int block_size,
                          const float* d_codebook, const void* d_x, int64_t ldx, int64_t n_tokens, const void* d_bias, int bias_dtype,
                          int activation, const int32_t* d_out_idx, const void* d_out_val, const int64_t* d_n_out, int64_t capacity, void* d_h,
                          int h_dtype, int64_t ldh, void* d_pre, int64_t ld_pre, int* d_status, void* d_ws, size_t ws_bytes, void* stream)
{
    const char* fn = "bof4_gated";
    if (ffn > INT32_MAX / 2) {
        set_error("%s: ffn must be below 2^30", fn);
        return BOF4_ERR_SHAPE;
    }
    LinearW w{};
    if (const int rc = linear_check(fn, &w, d_scales, scale_dtype, 2 * ffn, cols, block_size, n_tokens, activation, d_out_idx, d_out_val, d_n_out, capacity))
        return rc;
    if ((h_dtype != BOF4_F32 && h_dtype != BOF4_BF16) || (d_bias && bias_dtype != BOF4_F32 && bias_dtype != BOF4_BF16)) {
        set_error("%s: unknown dtype of h or bias", fn);
        return BOF4_ERR_DTYPE;
    }
    if (n_tokens > 1 && (ldx < cols || ldh < ffn || (d_pre && ld_pre < 2 * ffn))) {
        set_error("%s: a row stride is smaller than its row", fn);
        return BOF4_ERR_SHAPE;
    }
    if (!d_status) {
        set_error("%s: NULL status pointer", fn);
        return BOF4_ERR_INVALID_ARG;
    }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (ffn == 0 || n_tokens == 0) {
        BOF4_CUDA_TRY(cudaMemsetAsync(d_status, 0, sizeof(int), st));
        return BOF4_OK;
    }
    if (!d_h || (cols > 0 && (!d_codes || !d_scales || !d_codebook || !d_x))) {
        set_error("%s: NULL pointer", fn);
        return BOF4_ERR_INVALID_ARG;
    }
    if (n_tokens == 1) ldx = cols, ldh = ffn, ld_pre = 2 * ffn;
    LinearOut out{};
    out.bias = d_bias;
    out.bias_bf16 = bias_dtype == BOF4_BF16;
    out.y = d_h;
    out.ldy = ldh;
    out.y_bf16 = h_dtype == BOF4_BF16;
    out.pre = static_cast<uint16_t*>(d_pre);
    out.ld_pre = ld_pre;
    out.act = activation;
    out.n = ffn;
    out.tokens = n_tokens;
    out.gated = true;
    out.few_parts = true;
    out.set_alignment();
    if (cols == 0) {
        const int64_t want = (ffn * n_tokens + 255) / 256;
        launch_after(gated_empty_kernel, (int)(want < 8 * kSMs ? want : 8 * kSMs), 256, 0, st, out, d_status);
        BOF4_CUDA_TRY(cudaGetLastError());
        return BOF4_OK;
    }
    if (!aligned32(d_codes) || !aligned16(d_x) || ldx % 8) {
        set_error("%s: d_codes must be 32-byte aligned, d_x 16-byte aligned and ldx a multiple of 8", fn);
        return BOF4_ERR_INVALID_ARG;
    }
    GatedPlan p;
    if (!gated_plan(ffn, cols, n_tokens, false, h_dtype == BOF4_F32, w.capacity, &p)) {
        set_error("%s: matrix or batch too large", fn);
        return BOF4_ERR_SHAPE;
    }
    if (!d_ws || (reinterpret_cast<uintptr_t>(d_ws) & 255u) || ws_bytes < p.total) {
        set_error("%s: the workspace must be 256-byte aligned and hold %zu bytes", fn, p.total);
        return BOF4_ERR_WORKSPACE;
    }
    w.codes = d_codes;
    w.levels = d_codebook;
    if (!p.dense) {
        if (few_pays(w.rows, cols, n_tokens, w.capacity > 0)) return linear_few(fn, w, d_x, ldx, out, d_status, d_ws, ws_bytes, st);
        return linear_tc(fn, w, false, d_x, ldx, out, d_status, d_ws, ws_bytes, st);
    }
    unsigned char* const base = static_cast<unsigned char*>(d_ws);
    if (const int rc = gated_decode(w, base + p.w, st)) return rc;
    const DenseProduct q{d_x, ldx, base + p.w, 0, cols, w.rows, false, kDenseGated};
    DenseOut to{};
    to.y = d_h;
    to.ldy = ldh;
    to.n = ffn;
    to.tokens = n_tokens;
    to.y_bf16 = out.y_bf16;
    to.bias = d_bias;
    to.bias_bf16 = out.bias_bf16;
    to.pre = out.pre;
    to.ld_pre = ld_pre;
    to.act = activation;
    to.align = dense_align(d_h, ldh * (out.y_bf16 ? 2 : 4));
    to.pre_align = dense_align(d_pre, (ld_pre | ffn) * 2);
    return dense_product(fn, q, to, d_status, base, p.product, st);
}

extern "C" int bof4_gated_backward(const uint8_t* d_codes, const void* d_scales, int scale_dtype, int64_t ffn, int64_t cols, int block_size,
                                   const float* d_codebook, const void* d_dh, int dh_dtype, int64_t ld_dh, int64_t n_tokens, const void* d_pre,
                                   int64_t ld_pre, int activation, const int32_t* d_out_idx, const void* d_out_val, const int64_t* d_n_out,
                                   int64_t capacity, void* d_dx, int64_t ld_dx, float* d_dbias, int* d_status, void* d_ws, size_t ws_bytes, void* stream)
{
    const char* fn = "bof4_gated_backward";
    if (ffn > INT32_MAX / 2) {
        set_error("%s: ffn must be below 2^30", fn);
        return BOF4_ERR_SHAPE;
    }
    LinearW w{};
    if (const int rc = linear_check(fn, &w, d_scales, scale_dtype, 2 * ffn, cols, block_size, n_tokens, activation, d_out_idx, d_out_val, d_n_out, capacity))
        return rc;
    if (dh_dtype != BOF4_F32 && dh_dtype != BOF4_BF16) {
        set_error("%s: unknown dtype of dh", fn);
        return BOF4_ERR_DTYPE;
    }
    if (n_tokens > 1 && (ld_dh < ffn || (d_dx && ld_dx < cols) || ld_pre < 2 * ffn)) {
        set_error("%s: a row stride is smaller than its row", fn);
        return BOF4_ERR_SHAPE;
    }
    if (!d_status) {
        set_error("%s: NULL status pointer", fn);
        return BOF4_ERR_INVALID_ARG;
    }
    const bool nothing = ffn == 0 || n_tokens == 0, product = d_dx && cols > 0 && !nothing;
    if (!nothing && (!d_dh || !d_pre || (product && (!d_codes || !d_scales || !d_codebook)))) {
        set_error("%s: NULL pointer", fn);
        return BOF4_ERR_INVALID_ARG;
    }
    if (product && !aligned32(d_codes)) {
        set_error("%s: d_codes must be 32-byte aligned", fn);
        return BOF4_ERR_INVALID_ARG;
    }
    GatedPlan p{};
    const int col_blocks = (int)((ffn + kDzCols - 1) / kDzCols);
    if (!nothing && (!gated_plan(ffn, product ? cols : 0, n_tokens, true, false, w.capacity, &p) || p.chunks * col_blocks > INT32_MAX)) {
        set_error("%s: matrix or batch too large", fn);
        return BOF4_ERR_SHAPE;
    }
    if (!nothing && (!d_ws || (reinterpret_cast<uintptr_t>(d_ws) & 255u) || ws_bytes < p.total)) {
        set_error("%s: the workspace must be 256-byte aligned and hold %zu bytes", fn, p.total);
        return BOF4_ERR_WORKSPACE;
    }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!product) BOF4_CUDA_TRY(cudaMemsetAsync(d_status, 0, sizeof(int), st));  // (the product's kernel writes it)
    if (nothing) {  // sums over nothing
        if (d_dx && cols && n_tokens)
            BOF4_CUDA_TRY(cudaMemset2DAsync(d_dx, (size_t)(n_tokens > 1 ? ld_dx : cols) * 2, 0, (size_t)cols * 2, (size_t)n_tokens, st));
        if (d_dbias && ffn) BOF4_CUDA_TRY(cudaMemsetAsync(d_dbias, 0, (size_t)ffn * 8, st));
        return BOF4_OK;
    }
    if (!product && !d_dbias) return BOF4_OK;
    unsigned char* const base = static_cast<unsigned char*>(d_ws);
    if (n_tokens == 1) ld_dh = ffn, ld_pre = 2 * ffn, ld_dx = cols;
    uint16_t* const dz = reinterpret_cast<uint16_t*>(base + p.dz);
    float* const sums = p.chunks > 1 ? reinterpret_cast<float*>(base + p.sums) : d_dbias;
    const bool vec = aligned16(d_dh) && ld_dh % 8 == 0 && aligned16(d_pre) && ld_pre % 8 == 0 && ffn % 8 == 0;
    auto pick = [&](auto type) {
        using DT = decltype(type);
        if (vec) return d_dbias ? gated_dz_kernel<DT, true, true> : gated_dz_kernel<DT, false, true>;
        return d_dbias ? gated_dz_kernel<DT, true, false> : gated_dz_kernel<DT, false, false>;
    };
    launch_after(dh_dtype == BOF4_F32 ? pick(F32()) : pick(BF16()), (int)(p.chunks * col_blocks), 256, 0, st, d_dh, ld_dh, static_cast<const uint16_t*>(d_pre), ld_pre,
                 activation, ffn, n_tokens, product ? dz : nullptr, p.ld, d_dbias ? sums : nullptr, col_blocks, p.per);
    if (d_dbias && p.chunks > 1) linear_dbias(sums, 2 * ffn, p.chunks, d_dbias, st);
    BOF4_CUDA_TRY(cudaGetLastError());
    if (!product) return BOF4_OK;
    w.codes = d_codes;
    w.levels = d_codebook;
    if (p.dense) {
        if (const int rc = gated_decode(w, base + p.w, st)) return rc;
        const DenseProduct q{dz, p.ld, base + p.w, 0, w.rows, cols, true, kDenseStore};
        DenseOut to{};
        to.y = d_dx;
        to.ldy = ld_dx;
        to.n = cols;
        to.tokens = n_tokens;
        to.y_bf16 = true;
        to.align = dense_align(d_dx, ld_dx * 2);
        return dense_product(fn, q, to, d_status, base, p.product, st);
    }
    LinearOut out{};
    out.y = d_dx;
    out.ldy = ld_dx;
    out.y_bf16 = true;
    out.act = BOF4_ACT_NONE;
    out.n = cols;
    out.tokens = n_tokens;
    out.few_parts = true;
    out.set_alignment();
    return linear_tc(fn, w, true, dz, p.ld, out, d_status, base, p.product, st);
}
