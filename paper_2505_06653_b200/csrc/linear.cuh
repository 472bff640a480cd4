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
// act'(z) in fp32; far out, where the products below would be 0 * inf, the limits 0 and 1.
__device__ __forceinline__ float activate_slope(float z, int act)
{
    const float limit = z > 0.0f ? 1.0f : 0.0f;
    switch (act) {
        case BOF4_ACT_RELU: return z != z ? z : limit;
        case BOF4_ACT_GELU:
            if (fabsf(z) > 20.0f) return limit;
            return 0.5f * erfcf(-0.70710678118654752f * z) + z * 0.3989422804014327f * expf(-0.5f * z * z);
        case BOF4_ACT_GELU_TANH: {
            if (fabsf(z) > 12.0f) return limit;
            const float s = 1.0f / (1.0f + expf(-1.5957691216057308f * (z + 0.044715f * z * z * z)));
            return s + z * s * (1.0f - s) * 1.5957691216057308f * (1.0f + 0.134145f * z * z);
        }
        case BOF4_ACT_SILU: {
            if (fabsf(z) > 100.0f) return limit;
            const float s = 1.0f / (1.0f + expf(-z));
            return s + z * s * (1.0f - s);
        }
        default: return 1.0f;
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
bool linear_few_applies(int64_t rows, int64_t cols, int64_t tokens);
size_t linear_few_ws_bytes(int64_t rows, int64_t cols, int64_t tokens, int64_t capacity);
int linear_few(const char* who, const LinearW& w, const void* x, int64_t ldx, const LinearOut& out, int* status, void* ws, size_t ws_bytes,
               cudaStream_t st);

}  // namespace bof4
