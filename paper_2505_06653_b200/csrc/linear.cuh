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

// Where a sum goes: z = sum + bias (kept as bf16 where a backward pass will want it), y = act(z) + residual.  Element
// (t, o) of a matrix is at t * ld + o.
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
    void set_alignment()
    {
        const uintptr_t a = reinterpret_cast<uintptr_t>(y) | reinterpret_cast<uintptr_t>(residual) | reinterpret_cast<uintptr_t>(pre);
        const int64_t l = tokens > 1 ? ldy | (residual ? ld_residual : 0) | (pre ? ld_pre : 0) : 0;
        pairs = (a & 3u) == 0 && (l & 1) == 0;
        wide = (a & 15u) == 0 && (l & 7) == 0;
    }
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

// The tensor-core form: bytes of its workspace (0: too large), and the launch.  z[t, o] = sum_k operand[t, k] W^[o, k]
// (forward) or W^[k, o] (backward), then `out`.  operand: bf16, `ld` elements between tokens.
size_t linear_tc_ws_bytes(int64_t rows, int64_t cols, int64_t tokens, bool backward, int64_t capacity);
int linear_tc(const char* who, const LinearW& w, bool backward, const void* operand, int64_t ld, const LinearOut& out, int* status,
              void* ws, size_t ws_bytes, cudaStream_t st);

// The form for one to sixteen tokens.
bool linear_few_applies(int64_t rows, int64_t cols, int64_t tokens, bool list);
size_t linear_few_ws_bytes(int64_t rows, int64_t cols, int64_t tokens, int64_t capacity);
int linear_few(const char* who, const LinearW& w, const void* x, int64_t ldx, const LinearOut& out, int* status, void* ws, size_t ws_bytes,
               cudaStream_t st);

}  // namespace bof4
