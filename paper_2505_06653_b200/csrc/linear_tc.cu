// The host side of the products in linear_tc.cuh, lists of outliers, and the forward variants of the kernel.
#include "linear_tc.cuh"

namespace bof4 {

int linear_tc_forward(const LtLaunch& go) { return lt_launch<false, false>(go); }

// Outliers of a launch, as lists per k-block of a tile and producer warp: a node is {next, place in the warp's 32 x 64
// weights of the tile << 16 | value}.  Positions are distinct, so the order within a list does not matter.
__global__ void __launch_bounds__(256)
linear_outlier_lists(const int32_t* __restrict__ idx, const uint16_t* __restrict__ val, const int64_t* __restrict__ n_out, int64_t capacity,
                     int64_t rows, int64_t cols, bool backward, bool gated, int blocks, int* __restrict__ heads, int2* __restrict__ nodes)
{
    if (!after_previous()) return;
    int64_t end = *n_out;
    if (end > capacity) end = capacity;
    const int64_t n = rows * cols;
    for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < end; k += (int64_t)gridDim.x * 256) {
        const int64_t i = idx[k];
        if (i < 0 || i >= n) continue;
        const int row = (int)(i / cols), c = (int)(i - (int64_t)row * cols), ffn = (int)(rows >> 1);
        const int r = !gated ? row : row < ffn ? 2 * row : 2 * (row - ffn) + 1;  // gated tiles have gate and up rows in turn
        const int thread = backward ? (c >> 6 & 1) * 64 + (r & 63) : r & 127;
        const int64_t tile = backward ? c >> 7 : r >> 7, block = backward ? r >> 6 : c >> 6;
        const int next = atomicExch(heads + (tile * blocks + block) * 4 + (thread >> 5), (int)k);
        nodes[k] = make_int2(next, (int)((uint32_t)((thread & 31) << 6 | (c & 63)) << 16 | val[k]));
    }
}

// ---------------------------------------------------------------- host side

namespace {

struct LtPlan {
    LtWork work{};
    int ctas = 0, blocks = 0;
    int64_t tiles_m = 0;
    size_t parts = 0, heads = 0, nodes = 0, total = 0;  // byte offsets (the tickets are at 0), and the bytes of all
};

// False: too large for 32-bit line numbers.
bool lt_plan(int64_t rows, int64_t cols, int64_t tokens, bool backward, bool fp32, int64_t capacity, LtPlan* p, bool few_parts = false)
{
    const int64_t m = backward ? cols : rows, k = backward ? rows : cols;
    // (k-blocks past the end of K have zeros for the tokens)
    const int64_t tiles_m = (m + kLtM - 1) / kLtM, per_tile = (k + kLtK * kLtGroups - 1) / (kLtK * kLtGroups), blocks = per_tile * kLtGroups;
    // The tensor cores cut the sum off at every step of 16 of K, so the error grows with the steps in one accumulator: 3.6e-6 of the
    // result (2-norms) after K = 4096, 7e-6 after 8192.  That is nothing beside a rounding to bf16 (1.7e-3).  Results in fp32 with
    // a longer K have tiles of at most 128 tokens, which leave room for two accumulators that each take half of the steps (tiles
    // of 64 have four): 3.7e-6 at K = 8192, at 1.5 times the time (2048 tokens, 14336 rows: 660 us, 438 with tiles of 256).
    // Those of a gated block, and logits, go further (`segments` below).
    const int64_t widest = fp32 && k > kLtLongK ? 128 : kLtMaxN, most_n = (tokens + widest - 1) / widest;
    // the tokens are dealt evenly over the tiles, in multiples of 16
    const int64_t box = ((tokens + most_n - 1) / most_n + 15) & ~(int64_t)15, tiles_n = (tokens + box - 1) / box, tiles = tiles_m * tiles_n;
    if (tiles_m > (1 << 24) || tokens > 0x7fffff00 || k > 0x7fffff00 || tiles > 0x3fffffff || tiles * per_tile > 0x3fffffff) return false;
    LtWork& w = p->work;
    w.tiles = (int)tiles;
    w.tiles_n = (int)tiles_n;
    w.per_tile = (int)per_tile;
    w.box_n = (int)box;
    w.k = (int)k;
    // Four stages, and as many half lines of codes as there is room for beside them: four (256 tokens) to eight.  (Eight stages would leave
    // less than two lines of codes whatever the number of tokens: the table takes 64 KiB up to 64 of them, the stages themselves beyond.)
    w.table = box <= kLtTableN;
    const int room = kLtSmem - 1024 - (w.table ? kPairBytes : 0), stage = kLtABytes + (int)box * 128;
    w.halves = (room - kLtGroups * stage) / kLtHalfBytes & ~1;
    if (w.halves > kLtMaxHalves) w.halves = kLtMaxHalves;
    w.accs = box <= 64 ? 4 : box <= 128 ? 2 : 1;
    // Results in fp32 of a gated block, and logits: an accumulator takes at most 1024 of K, as in the form for many tokens (dense_tc.cu), and its sums are added in fp32: 0.7e-6
    // whatever K is, where one accumulator left 3e-6 at K = 4096.  That is more for the warps of the results than a segment of 256 tokens has time for: logits of 128256 rows by 256
    // tokens, K = 4096, 356 -> 383 us, gated 11008 x 4096 by 100 48.6 -> 51.6, by 256 62.7 -> 74.6.
    const bool segments = few_parts && fp32 && !backward;
    w.segment = segments ? kLtSegment * w.accs : (int)per_tile;
    // One CTA per SM, each with an equal part of the lines, but for few tiles of a long K: a tile is not cut into more than kLtMaxParts, which
    // one CTA adds up (128 x 256 sums in fp32 each).
    const int64_t lines = tiles * per_tile, most = tiles * kLtMaxParts;
    int64_t ctas = lines < kSMs ? lines : kSMs;
    if (ctas > most) ctas = most;
    if (few_parts && tiles < ctas) {
        // A line takes 1.7 us; a tile that is cut is written, waited for and read again, 2.5 us and 0.3 to 1.3 a part.  So a small matrix is not cut, and a few tiles
        // of a long K are not cut into all the CTAs there are, where equal parts of each tile save a seventh by this reckoning: gated 752 x 5568 by 201 tokens 38
        // us with every CTA at work, 31 this way; backward 3208 x 640 by 353 49 and 42.
        const double part = 0.3 + (double)box / 256.0, full = (double)lines / (double)ctas * 1.7 + 2.5 + ((double)ctas / (double)tiles + 1.0) * part;
        double best = 0.0;
        int64_t each = 0;
        for (int64_t j = 1; tiles * j <= ctas; ++j) {
            const double t = (double)((per_tile + j - 1) / j) * 1.7 + (j > 1 ? 2.5 + (double)j * part : 0.0);
            if (!each || t < best) best = t, each = j;
        }
        if (best < 0.85 * full) ctas = tiles * each;
    }
    p->ctas = (int)ctas;
    w.each = (int)(lines / ctas);
    w.extra = (int)(lines % ctas);
    p->blocks = (int)blocks;
    p->tiles_m = tiles_m;
    p->parts = up256((size_t)tiles * 8);
    p->heads = p->parts + up256((size_t)ctas * 2 * kLtM * box * 4);
    p->nodes = p->heads + (capacity > 0 ? up256((size_t)tiles_m * blocks * 16) : 0);
    p->total = p->nodes + (capacity > 0 ? up256((size_t)capacity * 8) : 0);
    return true;
}

}  // namespace

size_t linear_tc_ws_bytes(int64_t rows, int64_t cols, int64_t tokens, bool backward, int64_t capacity)
{
    LtPlan p, q;  // for results in bf16 and in fp32
    if (!lt_plan(rows, cols, tokens, backward, false, capacity, &p) || !lt_plan(rows, cols, tokens, backward, true, capacity, &q)) return 0;
    return p.total > q.total ? p.total : q.total;
}

int linear_tc(const char* who, const LinearW& w, bool backward, const void* operand, int64_t ld, const LinearOut& out, int* status,
              void* ws, size_t ws_bytes, cudaStream_t st)
{
    LtPlan p;
    const bool opq = w.out_idx && w.capacity > 0;
    if (!lt_plan(w.rows, w.cols, out.tokens, backward, !out.y_bf16, opq ? w.capacity : 0, &p, out.few_parts)) {
        set_error("%s: matrix or batch too large", who);
        return BOF4_ERR_SHAPE;
    }
    if (ws_bytes < p.total) {
        set_error("%s: the workspace has %zu bytes, %zu are needed", who, ws_bytes, p.total);
        return BOF4_ERR_WORKSPACE;
    }
    unsigned char* const base = static_cast<unsigned char*>(ws);
    p.work.epoch = tc_next_epoch();
    CUtensorMap code_map, token_map;
    int rc;
    const int64_t ffn = w.rows / 2;
    if ((rc = out.gated ? tc_make_map3(who, w.codes, 1, w.cols / 2, 2, ffn, ffn * (w.cols / 2), w.cols / 2, 64, 2, kLtM / 2, &code_map)
                        : tc_make_map(who, w.codes, 1, w.cols / 2, w.rows, w.cols / 2, 64, kLtM, &code_map)) ||
        (rc = tc_make_map(who, operand, 2, backward ? w.rows : w.cols, out.tokens, ld * 2, 128, p.work.box_n, &token_map)))
        return rc;
    int* heads = nullptr;
    int2* nodes = nullptr;
    if (opq) {
        heads = reinterpret_cast<int*>(base + p.heads);
        nodes = reinterpret_cast<int2*>(base + p.nodes);
        BOF4_CUDA_TRY(cudaMemsetAsync(heads, 0xff, (size_t)p.tiles_m * p.blocks * 16, st));
        const int64_t want = (w.capacity + 255) / 256;
        launch_after(linear_outlier_lists, (int)(want < 4 * kSMs ? want : 4 * kSMs), 256, 0, st, w.out_idx, w.out_val, w.n_out, w.capacity, w.rows,
                     w.cols, backward, out.gated, p.blocks, heads, nodes);
        BOF4_CUDA_TRY(cudaGetLastError());
    }
    const LtLaunch go{&code_map, &token_map, &w, &out, status, heads, nodes, &p.work, p.ctas, base, reinterpret_cast<float*>(base + p.parts), st};
    const bool segments = p.work.segment < p.work.per_tile;
    if (backward) rc = out.scale ? linear_tc_scaled(go) : linear_tc_backward(go);
    else if (out.gated) rc = segments ? linear_tc_gated_segments(go) : linear_tc_gated(go);
    else rc = segments ? linear_tc_forward_segments(go) : linear_tc_forward(go);
    if (rc) return rc;
    BOF4_CUDA_TRY(cudaGetLastError());
    return BOF4_OK;
}

}  // namespace bof4
