// Products of many tokens with a decoded matrix (bf16) on the tensor cores, and what becomes of the sums: the gated block, its
// gradient, and both products of the vocabulary loss.
#pragma once

#include "linear.cuh"
#include "tc.cuh"

namespace bof4 {

// What becomes of a tile of sums z[t, o].
enum DenseUse {
    kDenseStore,  // y[t, o] = z, bf16
    kDenseGated,  // y[t, f] = act(z[t, gate f]) * z[t, up f]; gate and up rows of B in turn
    kDenseGatedRows,  // the same where rows of y or pre do not begin at multiples of 32 bytes (chosen by dense_product)
    kDenseLoss,   // exponentials of logits against a reference per token, and their sums (cross_entropy.cu)
    kDenseAdd     // y[t, o] = y[t, o] * factor[t] + z, fp32
};

struct DenseOut {
    void* y;
    int64_t ldy, n, tokens;  // n: columns of z (gated: of y)
    bool y_bf16;
    int align, pre_align;    // bytes that rows of y (and both halves of those of pre) begin at multiples of, up to 32
    // gated
    const void* bias;        // [2 n] or NULL
    bool bias_bf16;
    uint16_t* pre;           // bf16 [t][2 n] or NULL
    int64_t ld_pre;
    int act;
    // loss: y holds the exponentials (NULL: not wanted), [t][ldy]
    const int64_t* targets;
    int64_t first_row;       // of the vocabulary in this piece
    const float* ref;        // [t]
    float2* stats;           // [column / 64][t]: the reference that was used, the sum
    float* target_logit;     // [t]
    // add
    const float* factor;     // [t], NULL: y is written, not added to
    bool first;              // loss: no reference yet, the guess is 0
    bool keep_status;        // *status is set where a wait runs out, and not cleared before
};

// The largest power of two up to 32 that divides an address and a distance in bytes.
inline int dense_align(const void* p, int64_t bytes)
{
    const uintptr_t all = reinterpret_cast<uintptr_t>(p) | (uintptr_t)bytes | 32u;
    return (int)(all & (~all + 1));
}

struct DenseWork {
    int tiles_m, tiles_n, per_tile;  // tiles of 256 tokens, of 256 columns of z, k-blocks of 64 of a tile
    int split, parts;                // the first `split` tiles are cut into so many parts along K, which are the first units of work
    int segment;                     // k-blocks of an accumulator
    int clusters;
    unsigned long long epoch;
};

// z[t, o] = sum_k a[t, k] B[o, k], or B[k, o] with n_major.  a: bf16, `lda` elements between tokens; b: bf16, rows without gaps.
struct DenseProduct {
    const void* a;
    int64_t lda;
    const void* b;
    int64_t ldb;   // elements between rows of b (0: k or n)
    int64_t k, n;  // n: rows of b (columns with n_major)
    bool n_major;
    DenseUse use;
};
size_t dense_ws_bytes(int64_t tokens, int64_t n, int64_t k);  // 0: too large
size_t dense_ws_most();                                       // of any sizes
int dense_product(const char* who, const DenseProduct& p, const DenseOut& out, int* status, void* ws, size_t ws_bytes, cudaStream_t st);

}  // namespace bof4
