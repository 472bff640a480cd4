// Entry points of bof4_linear and bof4_linear_backward, and the kernels beside the products: the gradient of the activation
// with the sums of the bias gradient, and the form without a product.
#include "linear.cuh"

namespace bof4 {

constexpr int kDzCols = 256;    // columns of a CTA: 32 lanes of eight
constexpr int kDzTokens = 32;   // tokens of a CTA, four a warp

// Eight values from column c of a row as they are in memory; those past the end are zero.
template <class T>
struct Dz8;
template <>
struct Dz8<BF16> {
    uint32_t w[4];
    __device__ __forceinline__ void load(const void* p, int64_t at, int count, bool vec)
    {
        const uint16_t* q = static_cast<const uint16_t*>(p) + at;
        if (vec) {
            const uint4 u = __ldg(reinterpret_cast<const uint4*>(q));
            w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                w[k] = (2 * k < count ? (uint32_t)__ldg(q + 2 * k) : 0u) | (2 * k + 1 < count ? (uint32_t)__ldg(q + 2 * k + 1) << 16 : 0u);
        }
    }
    __device__ __forceinline__ void values(float (&v)[8]) const
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[2 * k] = __uint_as_float(w[k] << 16), v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
    }
};
template <>
struct Dz8<F32> {
    float w[8];
    __device__ __forceinline__ void load(const void* p, int64_t at, int count, bool vec)
    {
        const float* q = static_cast<const float*>(p) + at;
        if (vec) {
            const float4 a = __ldg(reinterpret_cast<const float4*>(q)), b = __ldg(reinterpret_cast<const float4*>(q) + 1);
            w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) w[k] = k < count ? __ldg(q + k) : 0.0f;
        }
    }
    __device__ __forceinline__ void values(float (&v)[8]) const
    {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = w[k];
    }
};

// dz = dy * act'(pre), rounded to bf16 for the tensor cores, and the sums of the unrounded dz over a CTA's tokens.  One pass
// over dy and pre; a warp's four tokens are requested at once, and small CTAs leave a short last wave (2048 tokens of
// 14336 columns by SILU: 33 us, 5.3 TB/s; 64 tokens a CTA, two of a warp's at a time, and expf with rounded quotients took 67).  The tanh form
// takes 10 us more and GELU, whose erfc and exp are the rounded ones, 60: instructions bound them.
// Sums are added in a fixed order: tokens of a warp, the eight warps, and in dbias_kernel the CTAs' parts.
template <class DT>
__global__ void __launch_bounds__(256, DT::code == BOF4_F32 ? 2 : 4)
dz_kernel(const void* __restrict__ dy, int64_t ld_dy, const uint16_t* __restrict__ pre, int64_t ld_pre, int act, int64_t n, int64_t tokens,
          bool vec, uint16_t* __restrict__ dz, int64_t ld_dz, float* __restrict__ sums, int col_blocks)
{
    if (!after_previous()) return;
    __shared__ float s_sum[8][kDzCols + 4];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t chunk = blockIdx.x / col_blocks, c0 = (int64_t)(blockIdx.x % col_blocks) * kDzCols + lane * 8;
    const int count = (int)(n - c0 < 8 ? n - c0 : 8);
    const bool v8 = vec && count == 8;
    float sum[8] = {};
    if (count > 0) {
        constexpr int N = kDzTokens / 8;
        const int64_t t0 = chunk * kDzTokens + warp;
        Dz8<DT> a[N];
        Dz8<BF16> b[N];
#pragma unroll
        for (int u = 0; u < N; ++u) {
            if (t0 + 8 * u >= tokens) break;
            a[u].load(dy, (t0 + 8 * u) * ld_dy + c0, count, v8);
            if (pre) b[u].load(pre, (t0 + 8 * u) * ld_pre + c0, count, v8);
        }
#pragma unroll
        for (int u = 0; u < N; ++u) {
            if (t0 + 8 * u >= tokens) break;
            float g[8];
            a[u].values(g);
            if (pre) {
                float z[8];
                b[u].values(z);
                activate_slopes(g, z, act);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += g[k];  // (past the end of a row: zeros)
            if (dz) {
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = bf16_pair(g[2 * k], g[2 * k + 1]);
                *reinterpret_cast<uint4*>(dz + (t0 + 8 * u) * ld_dz + c0) = make_uint4(w[0], w[1], w[2], w[3]);  // rows of dz are padded to eight
            }
        }
    }
    if (!sums) return;
#pragma unroll
    for (int k = 0; k < 8; ++k) s_sum[warp][lane * 8 + k] = sum[k];
    __syncthreads();
    const int64_t c = (int64_t)(blockIdx.x % col_blocks) * kDzCols + threadIdx.x;
    if (c < n) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += s_sum[w][threadIdx.x];
        sums[chunk * n + c] = s;
    }
}

// The CTAs' parts of the bias gradient: 32 columns a CTA, every eighth part a warp.
__global__ void __launch_bounds__(256)
dbias_kernel(const float* __restrict__ sums, int64_t n, int64_t chunks, float* __restrict__ dbias)
{
    if (!after_previous()) return;
    __shared__ float s_sum[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (c < n) {
#pragma unroll 4
        for (int64_t k = warp; k < chunks; k += 8) s += __ldg(sums + k * n + c);
    }
    s_sum[warp][lane] = s;
    __syncthreads();
    if (warp || c >= n) return;
#pragma unroll
    for (int w = 1; w < 8; ++w) s += s_sum[w][lane];
    dbias[c] = s;
}

// The result where there is nothing to multiply (no columns).
__global__ void __launch_bounds__(256) linear_empty_kernel(const LinearOut out, int* __restrict__ status)
{
    if (!after_previous()) return;
    const int64_t total = out.tokens * out.n;
    if (blockIdx.x == 0 && threadIdx.x == 0) *status = 0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t t = i / out.n, o = i - t * out.n;
        out.store(0.0f, out.bias_at(o), out.residual_at(t, o), t, o);
    }
}

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// The checks that the two entry points share.
int linear_check(const char* fn, LinearW* w, const void* d_scales, int scale_dtype, int64_t rows, int64_t cols, int block_size, int64_t n_tokens,
                 int activation, const int32_t* d_out_idx, const void* d_out_val, const int64_t* d_n_out, int64_t capacity)
{
    if (rows < 0 || cols < 0 || n_tokens < 0) {
        set_error("%s: negative shape", fn);
        return BOF4_ERR_INVALID_ARG;
    }
    if (!valid_block_size(block_size) || cols % block_size) {
        set_error("%s: block_size must be a power of two in 32 ... 4096 that divides cols", fn);
        return BOF4_ERR_SHAPE;
    }
    if (rows > INT32_MAX || cols > INT32_MAX || n_tokens > INT32_MAX) {
        set_error("%s: rows, cols and n_tokens must be below 2^31", fn);
        return BOF4_ERR_SHAPE;
    }
    if (scale_dtype != BOF4_F32 && scale_dtype != BOF4_BF16) {
        set_error("%s: unknown scale dtype %d", fn, scale_dtype);
        return BOF4_ERR_DTYPE;
    }
    if (activation < BOF4_ACT_NONE || activation > BOF4_ACT_SILU) {
        set_error("%s: unknown activation %d", fn, activation);
        return BOF4_ERR_INVALID_ARG;
    }
    if (d_out_idx && (!d_out_val || !d_n_out)) {
        set_error("%s: outlier list needs d_out_idx, d_out_val and d_n_out together", fn);
        return BOF4_ERR_INVALID_ARG;
    }
    if (d_out_idx && (capacity < 0 || capacity > INT32_MAX)) {
        set_error("%s: outlier capacity negative or above 2^31 - 1", fn);
        return BOF4_ERR_CAPACITY;
    }
    if (d_out_idx && rows * cols > INT32_MAX) {
        set_error("%s: outlier indices are 32-bit, rows * cols must not exceed 2^31 - 1", fn);
        return BOF4_ERR_SHAPE;
    }
    w->scales = d_scales;
    w->rows = rows;
    w->cols = cols;
    w->block_size = block_size;
    w->scale_dtype = scale_dtype;
    w->block_shift = 0;
    while ((1 << w->block_shift) < block_size) ++w->block_shift;
    w->out_idx = d_out_idx;
    w->out_val = static_cast<const uint16_t*>(d_out_val);
    w->n_out = d_n_out;
    w->capacity = d_out_idx ? capacity : 0;
    return BOF4_OK;
}

// What the backward pass keeps behind the product's workspace: dz, then the sums of dz.
struct DzPlan {
    int64_t chunks, ld;
    size_t dz, sums, total;
};
DzPlan dz_plan(int64_t rows, int64_t tokens, size_t product)
{
    DzPlan p;
    p.chunks = (tokens + kDzTokens - 1) / kDzTokens;
    p.ld = (rows + 7) & ~(int64_t)7;
    p.dz = product;
    p.sums = p.dz + up256((size_t)tokens * p.ld * 2);
    p.total = p.sums + (p.chunks > 1 ? up256((size_t)p.chunks * rows * 4) : 0);
    return p;
}

}  // namespace
}  // namespace bof4

using namespace bof4;

extern "C" size_t bof4_linear_workspace_bytes(int64_t rows, int64_t cols, int64_t n_tokens, int backward, int64_t capacity)
{
    if (rows < 0 || cols < 0 || n_tokens < 0 || capacity < 0 || rows > INT32_MAX || cols > INT32_MAX || n_tokens > INT32_MAX || capacity > INT32_MAX)
        return 0;
    if (rows == 0 || n_tokens == 0) return 256;
    if (!backward && cols && linear_few_applies(rows, cols, n_tokens, capacity > 0)) return linear_few_ws_bytes(rows, cols, n_tokens, capacity);
    const size_t product = cols ? linear_tc_ws_bytes(rows, cols, n_tokens, backward != 0, capacity) : 256;
    if (!product || !backward) return product;
    return dz_plan(rows, n_tokens, product).total;
}

extern "C" int bof4_linear(const uint8_t* d_codes, const void* d_scales, int scale_dtype, int64_t rows, int64_t cols, int block_size,
                           const float* d_codebook, const void* d_x, int64_t ldx, int64_t n_tokens, const void* d_bias, int bias_dtype,
                           const void* d_residual, int64_t ld_residual, int activation, const int32_t* d_out_idx, const void* d_out_val,
                           const int64_t* d_n_out, int64_t capacity, void* d_y, int y_dtype, int64_t ldy, void* d_pre, int64_t ld_pre,
                           int* d_status, void* d_ws, size_t ws_bytes, void* stream)
{
    const char* fn = "bof4_linear";
    LinearW w{};
    if (const int rc = linear_check(fn, &w, d_scales, scale_dtype, rows, cols, block_size, n_tokens, activation, d_out_idx, d_out_val, d_n_out, capacity))
        return rc;
    if ((y_dtype != BOF4_F32 && y_dtype != BOF4_BF16) || (d_bias && bias_dtype != BOF4_F32 && bias_dtype != BOF4_BF16)) {
        set_error("%s: unknown dtype of y or bias", fn);
        return BOF4_ERR_DTYPE;
    }
    if (n_tokens > 1 && (ldx < cols || ldy < rows || (d_residual && ld_residual < rows) || (d_pre && ld_pre < rows))) {
        set_error("%s: a row stride is smaller than its row", fn);
        return BOF4_ERR_SHAPE;
    }
    if (!d_status) {
        set_error("%s: NULL status pointer", fn);
        return BOF4_ERR_INVALID_ARG;
    }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rows == 0 || n_tokens == 0) {
        BOF4_CUDA_TRY(cudaMemsetAsync(d_status, 0, sizeof(int), st));
        return BOF4_OK;
    }
    if (!d_y || (cols > 0 && (!d_codes || !d_scales || !d_codebook || !d_x))) {
        set_error("%s: NULL pointer", fn);
        return BOF4_ERR_INVALID_ARG;
    }
    LinearOut out{};
    out.bias = d_bias;
    out.bias_bf16 = bias_dtype == BOF4_BF16;
    out.residual = d_residual;
    out.ld_residual = ld_residual;
    out.y = d_y;
    out.ldy = ldy;
    out.y_bf16 = y_dtype == BOF4_BF16;
    out.pre = static_cast<uint16_t*>(d_pre);
    out.ld_pre = ld_pre;
    out.act = activation;
    out.n = rows;
    out.tokens = n_tokens;
    out.set_alignment();
    if (cols == 0) {
        const int64_t want = (rows * n_tokens + 255) / 256;
        launch_after(linear_empty_kernel, (int)(want < 8 * kSMs ? want : 8 * kSMs), 256, 0, st, out, d_status);
        BOF4_CUDA_TRY(cudaGetLastError());
        return BOF4_OK;
    }
    if (n_tokens == 1) ldx = cols;
    if (!aligned32(d_codes) || !aligned16(d_x) || ldx % 8) {
        set_error("%s: d_codes must be 32-byte aligned, d_x 16-byte aligned and ldx a multiple of 8", fn);
        return BOF4_ERR_INVALID_ARG;
    }
    if (!d_ws || (reinterpret_cast<uintptr_t>(d_ws) & 255u)) {
        set_error("%s: the workspace must be 256-byte aligned", fn);
        return BOF4_ERR_WORKSPACE;
    }
    w.codes = d_codes;
    w.levels = d_codebook;
    if (linear_few_applies(rows, cols, n_tokens, w.capacity > 0)) return linear_few(fn, w, d_x, ldx, out, d_status, d_ws, ws_bytes, st);
    return linear_tc(fn, w, false, d_x, ldx, out, d_status, d_ws, ws_bytes, st);
}

extern "C" int bof4_linear_backward(const uint8_t* d_codes, const void* d_scales, int scale_dtype, int64_t rows, int64_t cols, int block_size,
                                    const float* d_codebook, const void* d_dy, int dy_dtype, int64_t ld_dy, int64_t n_tokens,
                                    const void* d_pre, int64_t ld_pre, int activation, const int32_t* d_out_idx, const void* d_out_val,
                                    const int64_t* d_n_out, int64_t capacity, void* d_dx, int64_t ld_dx, float* d_dbias, int* d_status,
                                    void* d_ws, size_t ws_bytes, void* stream)
{
    const char* fn = "bof4_linear_backward";
    LinearW w{};
    if (const int rc = linear_check(fn, &w, d_scales, scale_dtype, rows, cols, block_size, n_tokens, activation, d_out_idx, d_out_val, d_n_out, capacity))
        return rc;
    if (dy_dtype != BOF4_F32 && dy_dtype != BOF4_BF16) {
        set_error("%s: unknown dtype of dy", fn);
        return BOF4_ERR_DTYPE;
    }
    const bool slope = activation != BOF4_ACT_NONE;
    if (n_tokens > 1 && (ld_dy < rows || (d_dx && ld_dx < cols) || (slope && d_pre && ld_pre < rows))) {
        set_error("%s: a row stride is smaller than its row", fn);
        return BOF4_ERR_SHAPE;
    }
    if (!d_status) {
        set_error("%s: NULL status pointer", fn);
        return BOF4_ERR_INVALID_ARG;
    }
    const bool nothing = rows == 0 || n_tokens == 0, product = d_dx && cols > 0 && !nothing;
    if (!nothing && (!d_dy || (slope && !d_pre) || (product && (!d_codes || !d_scales || !d_codebook)))) {
        set_error("%s: NULL pointer (an activation needs the values before it, d_pre)", fn);
        return BOF4_ERR_INVALID_ARG;
    }
    if (product && !aligned32(d_codes)) {
        set_error("%s: d_codes must be 32-byte aligned", fn);
        return BOF4_ERR_INVALID_ARG;
    }
    const size_t need_product = product ? linear_tc_ws_bytes(rows, cols, n_tokens, true, w.capacity) : 0;
    const DzPlan plan = dz_plan(rows, n_tokens, need_product);
    const int col_blocks = (int)((rows + kDzCols - 1) / kDzCols);
    if ((product && !need_product) || plan.chunks * col_blocks > INT32_MAX) {
        set_error("%s: matrix or batch too large", fn);
        return BOF4_ERR_SHAPE;
    }
    if (!nothing && (!d_ws || (reinterpret_cast<uintptr_t>(d_ws) & 255u) || ws_bytes < plan.total)) {
        set_error("%s: the workspace must be 256-byte aligned and hold %zu bytes", fn, plan.total);
        return BOF4_ERR_WORKSPACE;
    }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!product) BOF4_CUDA_TRY(cudaMemsetAsync(d_status, 0, sizeof(int), st));  // (the product's kernel writes it)
    if (nothing) {  // sums over nothing
        if (d_dx && cols && n_tokens)
            BOF4_CUDA_TRY(cudaMemset2DAsync(d_dx, (size_t)(n_tokens > 1 ? ld_dx : cols) * 2, 0, (size_t)cols * 2, (size_t)n_tokens, st));
        if (d_dbias && rows) BOF4_CUDA_TRY(cudaMemsetAsync(d_dbias, 0, (size_t)rows * 4, st));
        return BOF4_OK;
    }
    unsigned char* const base = static_cast<unsigned char*>(d_ws);
    const uint16_t* const pre = slope ? static_cast<const uint16_t*>(d_pre) : nullptr;
    if (n_tokens == 1) ld_dy = ld_pre = rows;
    // dy itself is the operand where nothing has to be done to it and TMA can read it
    const bool direct = !pre && dy_dtype == BOF4_BF16 && aligned16(d_dy) && ld_dy % 8 == 0, make_dz = product && !direct;
    uint16_t* const dz = reinterpret_cast<uint16_t*>(base + plan.dz);
    float* const sums = plan.chunks > 1 ? reinterpret_cast<float*>(base + plan.sums) : d_dbias;
    if (make_dz || d_dbias) {
        const bool vec = aligned16(d_dy) && ld_dy % 8 == 0 && (!pre || (aligned16(pre) && ld_pre % 8 == 0));
        launch_after(dy_dtype == BOF4_F32 ? dz_kernel<F32> : dz_kernel<BF16>, (int)(plan.chunks * col_blocks), 256, 0, st, d_dy, ld_dy, pre, ld_pre,
                     activation, rows, n_tokens, vec, make_dz ? dz : nullptr, plan.ld, d_dbias ? sums : nullptr, col_blocks);
        if (d_dbias && plan.chunks > 1) launch_after(dbias_kernel, (int)((rows + 31) / 32), 256, 0, st, sums, rows, plan.chunks, d_dbias);
        BOF4_CUDA_TRY(cudaGetLastError());
    }
    if (!product) return BOF4_OK;
    w.codes = d_codes;
    w.levels = d_codebook;
    LinearOut out{};
    out.y = d_dx;
    out.ldy = n_tokens > 1 ? ld_dx : cols;
    out.y_bf16 = true;
    out.act = BOF4_ACT_NONE;
    out.n = cols;
    out.tokens = n_tokens;
    out.set_alignment();
    return linear_tc(fn, w, true, direct ? d_dy : dz, direct ? ld_dy : plan.ld, out, d_status, d_ws, need_product, st);
}
