// What the kernels of bof4_linear, bof4_linear_backward and bof4_moe share: activations and their derivatives, and what
// becomes of a sum (bias, activation, residual, rounding).
#pragma once

#include "common.cuh"

namespace bof4 {

__device__ __forceinline__ float bf16_value(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ uint16_t bf16_round(float v)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(0.0f), "f"(v));
    return (uint16_t)r;
}

// act(z) in fp32.  GELU by the complementary error function, which keeps its relative precision where the weight of z is
// small; the tanh form as z * sigmoid(2 u), which is the same function without a cancelling 1 + tanh.
__device__ __forceinline__ float activate(float z, int act)
{
    switch (act) {
        case BOF4_ACT_RELU: return z <= 0.0f ? 0.0f : z;
        case BOF4_ACT_GELU: return 0.5f * z * erfcf(-0.70710678118654752f * z);
        case BOF4_ACT_GELU_TANH: return z / (1.0f + expf(-1.5957691216057308f * (z + 0.044715f * z * z * z)));
        case BOF4_ACT_SILU: return z / (1.0f + expf(-z));
        default: return z;
    }
}
// The same for several values: one branch for all of them.
template <int N>
__device__ __forceinline__ void activate_all(float (&z)[N], int act)
{
    switch (act) {
        case BOF4_ACT_RELU:
#pragma unroll
            for (int k = 0; k < N; ++k) z[k] = activate(z[k], BOF4_ACT_RELU);
            break;
        case BOF4_ACT_GELU:
#pragma unroll
            for (int k = 0; k < N; ++k) z[k] = activate(z[k], BOF4_ACT_GELU);
            break;
        case BOF4_ACT_GELU_TANH:
#pragma unroll
            for (int k = 0; k < N; ++k) z[k] = activate(z[k], BOF4_ACT_GELU_TANH);
            break;
        case BOF4_ACT_SILU:
#pragma unroll
            for (int k = 0; k < N; ++k) z[k] = activate(z[k], BOF4_ACT_SILU);
            break;
        default: break;
    }
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// act'(z) in fp32; far out, where the products below would be 0 * inf, the limits 0 and 1.  The logistic part s(v) = 1 / (1 + exp(-v)) and its
// slope s (1 - s) come from t = exp(-|v|), which neither overflows nor leaves a 1 - s to cancel: s(|v|) = 1 / (1 + t), s(-|v|) = t / (1 + t).
// The quotient is off by two units in the last place and t by 2 + 1.2 |v| of its own (half of the instructions of the rounded forms); with all
// roundings a slope is within 2^-20 (the argument is beside test_slopes; over all bf16 values at most 1.9e-7, where s + z s (1 - s) as it
// stands was off by up to 1.9e-6 at z = 5 of the tanh form).
__device__ __forceinline__ float activate_slope(float z, int act)
{
    const float limit = z > 0.0f ? 1.0f : 0.0f;
    switch (act) {
        case BOF4_ACT_RELU: return z != z ? z : limit;
        case BOF4_ACT_GELU: {
            const float v = 0.5f * erfcf(-0.70710678118654752f * z) + z * 0.3989422804014327f * expf(-0.5f * z * z);
            return fabsf(z) > 20.0f ? limit : v;
        }
        case BOF4_ACT_GELU_TANH: {
            const float v = 1.5957691216057308f * (z + 0.044715f * z * z * z), t = __expf(-fabsf(v)), big = __fdividef(1.0f, 1.0f + t), little = t * big;
            const float d = (z > 0.0f ? big : little) + z * (1.5957691216057308f * (1.0f + 0.134145f * z * z)) * (big * little);
            return fabsf(z) > 12.0f ? limit : d;
        }
        case BOF4_ACT_SILU: {
            const float t = __expf(-fabsf(z)), big = __fdividef(1.0f, 1.0f + t), little = t * big;
            const float d = (z > 0.0f ? big : little) + z * (big * little);
            return fabsf(z) > 100.0f ? limit : d;
        }
        default: return 1.0f;
    }
}
// g *= act'(z) for several values: one branch for all of them.
template <int N>
__device__ __forceinline__ void activate_slopes(float (&g)[N], const float (&z)[N], int act)
{
    switch (act) {
        case BOF4_ACT_RELU:
#pragma unroll
            for (int k = 0; k < N; ++k) g[k] *= activate_slope(z[k], BOF4_ACT_RELU);
            break;
        case BOF4_ACT_GELU:
#pragma unroll
            for (int k = 0; k < N; ++k) g[k] *= activate_slope(z[k], BOF4_ACT_GELU);
            break;
        case BOF4_ACT_GELU_TANH:
#pragma unroll
            for (int k = 0; k < N; ++k) g[k] *= activate_slope(z[k], BOF4_ACT_GELU_TANH);
            break;
        case BOF4_ACT_SILU:
#pragma unroll
            for (int k = 0; k < N; ++k) g[k] *= activate_slope(z[k], BOF4_ACT_SILU);
            break;
        default: break;
    }
}

// act(z) for the gated block: the logistic forms with half of the instructions, within 2^-20 |z| (the argument is beside test_activations_at_every_value).  Relative to the result,
// which falls off like e^v with v the exponential's argument, that is a precision that falls with |v|: the exponential is off by 2 + 1.2 |v| units and, in the tanh form, v itself by up
// to two, which is |v| times as many of the result's; where e^-v is above 2^126 the quotient is zero.  (Its results' warps are waited for at the end of a launch: 256 tokens of 11008 x 4096 took 78 us
// with the rounded quotient and exponential.)
template <int N>
__device__ __forceinline__ void activate_gate(float (&z)[N], int act)
{
    if (act == BOF4_ACT_SILU) {
#pragma unroll
        for (int k = 0; k < N; ++k) z[k] *= __fdividef(1.0f, 1.0f + __expf(-z[k]));
    } else if (act == BOF4_ACT_GELU_TANH) {
#pragma unroll
        for (int k = 0; k < N; ++k) z[k] *= __fdividef(1.0f, 1.0f + __expf(-1.5957691216057308f * (z[k] + 0.044715f * z[k] * z[k] * z[k])));
    } else {
        activate_all(z, act);
    }
}
// act(z) and act'(z) together: the logistic and the normal distribution's part is evaluated once (accurate as above).
__device__ __forceinline__ void activate_both(float z, int act, float& a, float& slope)
{
    switch (act) {
        case BOF4_ACT_RELU: a = activate(z, BOF4_ACT_RELU), slope = activate_slope(z, BOF4_ACT_RELU); break;
        case BOF4_ACT_GELU: {
            const float cdf = 0.5f * erfcf(-0.70710678118654752f * z), d = cdf + z * 0.3989422804014327f * expf(-0.5f * z * z);
            a = z * cdf, slope = fabsf(z) > 20.0f ? (z > 0.0f ? 1.0f : 0.0f) : d;
            break;
        }
        case BOF4_ACT_GELU_TANH: {
            const float v = 1.5957691216057308f * (z + 0.044715f * z * z * z), t = __expf(-fabsf(v)), big = __fdividef(1.0f, 1.0f + t), little = t * big;
            const float s = z > 0.0f ? big : little, d = s + z * (1.5957691216057308f * (1.0f + 0.134145f * z * z)) * (big * little);
            a = z * s, slope = fabsf(z) > 12.0f ? (z > 0.0f ? 1.0f : 0.0f) : d;
            break;
        }
        case BOF4_ACT_SILU: {
            const float t = __expf(-fabsf(z)), big = __fdividef(1.0f, 1.0f + t), little = t * big, s = z > 0.0f ? big : little;
            a = z * s, slope = fabsf(z) > 100.0f ? (z > 0.0f ? 1.0f : 0.0f) : s + z * (big * little);
            break;
        }
        default: a = z, slope = 1.0f;
    }
}

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

// Where a sum goes: z = sum + bias (kept as bf16 where a backward pass will want it), y = act(z) + residual.  Element
// (t, o) of a matrix is at t * ld + o.  Gated: n columns f of y, for which z has 2 n, y = act(z[f]) * z[n + f]; bias and pre hold 2 n too.
struct LinearOut {
    const void* bias;      // [n] or NULL
    const void* residual;  // type of y, or NULL
    uint16_t* pre;         // bf16, or NULL
    void* y;
    int64_t ld_residual, ld_pre, ldy, n, tokens;
    int act;
    bool bias_bf16, y_bf16;
    // rows of y, residual and pre begin at addresses that hold pairs of bf16 values / 16 bytes of their type
    bool pairs, wide;
    const float* scale;  // backward: what the sums of a token are multiplied by, or NULL
    bool gated;
    bool few_parts;    // tiles are cut along K only as far as it pays (gated, loss)
    bool keep_status;  // *status is set where a wait runs out, and not cleared before
    void set_alignment()
    {
        const uintptr_t a = reinterpret_cast<uintptr_t>(y) | reinterpret_cast<uintptr_t>(residual) | reinterpret_cast<uintptr_t>(pre);
        const int64_t l = tokens > 1 ? ldy | (residual ? ld_residual : 0) | (pre ? ld_pre : 0) : 0;
        pairs = (a & 3u) == 0 && (l & 1) == 0;
        wide = (a & 15u) == 0 && (l & 7) == 0;
    }
    // A scale of zero is an ignored token's: nothing of its sums is wanted, whatever weights that are not finite have made of them.
    static __device__ __forceinline__ float scaled(float sum, float f) { return f == 0.0f ? 0.0f : sum * f; }
    __device__ __forceinline__ float bias_at(int64_t o) const
    {
        if (!bias) return 0.0f;
        return bias_bf16 ? bf16_value(__ldg(static_cast<const uint16_t*>(bias) + o)) : __ldg(static_cast<const float*>(bias) + o);
    }
    // (the residual may be y itself: plain loads)
    __device__ __forceinline__ float residual_at(int64_t t, int64_t o) const
    {
        if (!residual) return 0.0f;
        const int64_t i = t * ld_residual + o;
        return y_bf16 ? bf16_value(*(static_cast<const uint16_t*>(residual) + i)) : *(static_cast<const float*>(residual) + i);
    }
    __device__ __forceinline__ void store(float sum, float b, float r, int64_t t, int64_t o) const
    {
        const float z = sum + b;
        if (pre) pre[t * ld_pre + o] = bf16_round(z);
        const float v = activate(z, act) + r;
        if (y_bf16) static_cast<uint16_t*>(y)[t * ldy + o] = bf16_round(v);
        else static_cast<float*>(y)[t * ldy + o] = v;
    }
    // gated: the sums of columns f and n + f
    __device__ __forceinline__ void store_pair(float g, float u, int64_t t, int64_t f) const
    {
        g += bias_at(f), u += bias_at(n + f);
        if (pre) pre[t * ld_pre + f] = bf16_round(g), pre[t * ld_pre + n + f] = bf16_round(u);
        float v[1] = {g};
        activate_gate(v, act);
        v[0] *= u;
        if (y_bf16) static_cast<uint16_t*>(y)[t * ldy + f] = bf16_round(v[0]);
        else static_cast<float*>(y)[t * ldy + f] = v[0];
    }
    // of columns f and f + 1 (f even)
    __device__ __forceinline__ void store_pairs(const float4& z, int64_t t, int64_t f) const
    {
        if (!(pairs && y_bf16 && f + 1 < n && (!pre || (n & 1) == 0))) {
            if (f < n) store_pair(z.x, z.y, t, f);
            if (f + 1 < n) store_pair(z.z, z.w, t, f + 1);
            return;
        }
        float g[2] = {z.x + bias_at(f), z.z + bias_at(f + 1)}, u[2] = {z.y + bias_at(n + f), z.w + bias_at(n + f + 1)};
        if (pre) {
            *reinterpret_cast<uint32_t*>(pre + t * ld_pre + f) = bf16_pair(g[0], g[1]);
            *reinterpret_cast<uint32_t*>(pre + t * ld_pre + n + f) = bf16_pair(u[0], u[1]);
        }
        activate_gate(g, act);
        *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(y) + t * ldy + f) = bf16_pair(g[0] * u[0], g[1] * u[1]);
    }
};

// Sums of four neighbouring rows o ... o + 3 (o a multiple of four) of a token: residual (loaded before), bias, store.
struct LinearFour {
    float r[4];
    __device__ __forceinline__ void residual(const LinearOut& out, int64_t t, int64_t o)
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) r[k] = 0.0f;
        if (!out.residual) return;
        const int64_t i = t * out.ld_residual + o;
        if (out.wide && o + 3 < out.n) {
            if (out.y_bf16) {
                const uint2 u = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(out.residual) + i);
                r[0] = __uint_as_float(u.x << 16), r[1] = __uint_as_float(u.x & 0xffff0000u), r[2] = __uint_as_float(u.y << 16), r[3] = __uint_as_float(u.y & 0xffff0000u);
            } else {
                const float4 v = *reinterpret_cast<const float4*>(static_cast<const float*>(out.residual) + i);
                r[0] = v.x, r[1] = v.y, r[2] = v.z, r[3] = v.w;
            }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (o + k < out.n) r[k] = out.residual_at(t, o + k);
        }
    }
    __device__ __forceinline__ void store(const LinearOut& out, const float4& sum, int64_t t, int64_t o) const
    {
        float z[4] = {sum.x, sum.y, sum.z, sum.w};
        if (out.bias) {
#pragma unroll
            for (int k = 0; k < 4; ++k) z[k] += o + k < out.n ? out.bias_at(o + k) : 0.0f;
        }
        if (!(out.wide && o + 3 < out.n)) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (o + k < out.n) out.store(z[k], 0.0f, r[k], t, o + k);
            return;
        }
        if (out.pre) *reinterpret_cast<uint2*>(out.pre + t * out.ld_pre + o) = make_uint2(bf16_pair(z[0], z[1]), bf16_pair(z[2], z[3]));
        activate_all(z, out.act);
#pragma unroll
        for (int k = 0; k < 4; ++k) z[k] += r[k];
        if (out.y_bf16) *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out.y) + t * out.ldy + o) = make_uint2(bf16_pair(z[0], z[1]), bf16_pair(z[2], z[3]));
        else *reinterpret_cast<float4*>(static_cast<float*>(out.y) + t * out.ldy + o) = make_float4(z[0], z[1], z[2], z[3]);
    }
};

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Parts of a workspace begin at multiples of 256 bytes.
inline size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }

// The 4-bit matrix and its outlier list.
struct LinearW {
    const uint8_t* codes;
    const void* scales;
    const float* levels;
    int64_t rows, cols;
    int block_size, block_shift, scale_dtype;
    const int32_t* out_idx;   // NULL without a list
    const uint16_t* out_val;
    const int64_t* n_out;
    int64_t capacity;
};

// The checks that the entry points share; fills *w but for codes and levels.
int linear_check(const char* fn, LinearW* w, const void* d_scales, int scale_dtype, int64_t rows, int64_t cols, int block_size, int64_t n_tokens,
                 int activation, const int32_t* d_out_idx, const void* d_out_val, const int64_t* d_n_out, int64_t capacity);
constexpr int kDzCols = 256;    // columns of a CTA that forms gradients of activations: 32 lanes of eight
constexpr int kDzTokens = 32;   // its tokens, four a warp
void linear_dbias(const float* sums, int64_t n, int64_t chunks, float* dbias, cudaStream_t st);

// The tensor-core form: bytes of its workspace (0: too large), and the launch.  z[t, o] = sum_k operand[t, k] W^[o, k]
// (forward) or W^[k, o] (backward), then `out`.  operand: bf16, `ld` elements between tokens.
size_t linear_tc_ws_bytes(int64_t rows, int64_t cols, int64_t tokens, bool backward, int64_t capacity);
int linear_tc(const char* who, const LinearW& w, bool backward, const void* operand, int64_t ld, const LinearOut& out, int* status,
              void* ws, size_t ws_bytes, cudaStream_t st);

// The form for one to sixteen tokens.
bool linear_few_applies(int64_t rows, int64_t cols, int64_t tokens, bool list);
size_t linear_few_ws_bytes(int64_t rows, int64_t cols, int64_t tokens, int64_t capacity, bool few_parts = false);
int linear_few(const char* who, const LinearW& w, const void* x, int64_t ldx, const LinearOut& out, int* status, void* ws, size_t ws_bytes,
               cudaStream_t st);
// Where it pays in a gated block or a loss: in large matrices up to twelve tokens only (28672 x 8192 gated by 12 164 us against 158, by 16 186 against 158;
// 11008 x 4096 by 12 42 against 45, by 16 47 against 45).
inline bool few_pays(int64_t rows, int64_t cols, int64_t tokens, bool list)
{
    return linear_few_applies(rows, cols, tokens, list) && !(tokens > 12 && rows * cols >= (int64_t)1 << 26);
}

}  // namespace bof4
