// The 16-bit product with its fused epilogues as the other translation units call it (see dense_gemm_kernel.cuh).
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace mxfp4 {

enum DenseEpilogue { kDenseStore, kDenseScaled, kDenseGated, kDensePartials, kDenseLogitGrad };
enum DenseOut { kDenseBf16, kDenseF32, kDenseAddF32 };

// What one operand's panel may take of L2.  The order decides how much is read from memory, which costs energy, and the power
// cap makes that time: loss of 8192 tokens, pass after pass, 6250 us with bands of columns only and no hints, 6130 with
// bands of rows where that reads less, 6060 with cache hints; gated forward pass 1470, 1450 and 1425.  Panels of 16, 24, 48
// and 68 MB: 6400, 6330, 6340 and 6520 where 32 took 6220.
constexpr int64_t kDensePanelBytes = int64_t{32} << 20;
constexpr int64_t kDenseMaxDim = 0x7FFFFF00;
constexpr int64_t kDenseMaxK = (int64_t{1} << 30) - 64;      // of all segments: positions along K, and steps past them, fit 32 bits
constexpr int kDensePairs = 74;  // work is shared out for the pairs of CTAs of this many SMs, whatever the device has

// Sizes of one product as the kernel needs them.
struct DenseShape {
    int32_t M, N, K;             // of one segment; gated: N features of each projection
    int32_t tiles_m, tiles_n;    // of all segments
    int32_t seg_tiles_m;
    int32_t k_steps;             // of all segments
    int32_t seg_k_steps;
    int32_t width;               // rows of B per CTA and tile: a tile has 2 * width columns
    int32_t band;                // tile columns (band_m: rows) per band of the tile order
    int32_t band_m;
    int32_t hints;               // the panel is kept in L2, what passes it is not
    int32_t splits;              // pieces along K, each with an output of its own
    int32_t split_rows;          // output rows from one piece's to the next one's
    int32_t items;               // tiles * splits
    int32_t a_mn;                // A is stored along its own rows
    int32_t out;                 // DenseOut
};

// What the epilogues read.
struct DenseExtra {
    int32_t act;                 // gated
    int32_t keep;                // g and u are stored too
    __nv_bfloat16* out[3];       // h, g, u, for the parts of tiles that are not whole boxes
    int64_t ld_out[3];
    // log probabilities: columns col_base .. col_base + N of `vocab`
    float scale;
    int32_t ld_grad;             // columns of the gradient's buffer, those past N set to 0
    int32_t rows;                // gradient of the logits, and products of it: positions (see dense_common)
    int64_t vocab, col_base;
    const int64_t* targets;
    const float* lse;
    const float* d_logp;
    const float* d_lse;
    float2* parts;               // [ceil(N / width)][ld_parts]: maximum, sum of exponentials
    int64_t ld_parts;
    float* picked;               // the target's value
};

struct DenseParams {
    DenseShape q[2];             // a launch's products
    DenseExtra x;
};

struct DenseMatrix {
    const void* p;
    int64_t ld;                  // elements
};

// a and b are stored along K, or (a_mn, b_mn) along their own rows: [K x M], [K x N].  `stack_m`: two matrices a, each with
// its own output; `stack_k`: two pairs (a, b) whose products are added.  splits > 1 (not with stack_m): out[0] has
// dense_split_rows(M) rows per piece.
struct DenseProduct {
    int64_t M = 0, N = 0, K = 0;
    bool a_mn = false, b_mn = false;
    bool stack_m = false, stack_k = false;
    int splits = 1;
    DenseOut kind = kDenseBf16;
    DenseMatrix a[2] = {}, b[2] = {}, out[3] = {};
};

// One launch of one or two products with plain outputs (b stored along its rows), or of one with another epilogue.
// `extra`: of the gradient of the logits that the products are of; NULL for others.
int dense_store(const DenseProduct* products, int n, const DenseExtra* extra, int sm_count, cudaStream_t st);
int dense_fused(DenseEpilogue epilogue, const DenseProduct& product, const DenseExtra& extra, int sm_count, cudaStream_t st);

// The sum of `pieces` products of splits as dense_store leaves them, to bf16; cols a multiple of 8.
int dense_round(const float* from, int pieces, int64_t rows, int64_t cols, void* to, int64_t ld, int sm_count, cudaStream_t st);

inline int64_t dense_tiles(int64_t n, int64_t tile) { return (n + tile - 1) / tile; }
inline int64_t dense_split_rows(int64_t M) { return dense_tiles(M, 256) * 256; }

// Columns per CTA and tile of a product with few rows (64 to 128, a multiple of 8; `per_tile`: 1 or 2 of these widths side by side
// make a tile's columns): 224 tiles are three rounds of the pairs and two tiles more, where narrower ones make
// four even rounds.  A step costs a tile its columns and about 32 more.
inline int dense_width(int64_t M, int64_t N, int per_tile)
{
    int best = 128;
    int64_t least = 0;
    for (int w = 128; w >= 64; w -= 8) {
        const int64_t cost = dense_tiles(dense_tiles(M, 256) * dense_tiles(N, w * per_tile), kDensePairs) * (w + 32);
        if (w == 128) least = cost * 19 / 20;       // full width unless it costs a twentieth more
        else if (cost < least) {
            least = cost;
            best = w;
        }
    }
    return best;
}

// Pieces along K for a product of few tiles: as many as keep the pairs busiest, none shorter than eight steps of 64; a piece
// costs about eight steps besides its own.  With
// more tiles than pairs a tile stays whole; what a last, partial wave leaves idle is filled by a launch's other product.
inline int dense_splits(int64_t M, int64_t N, int64_t K_all)
{
    const int64_t tiles = dense_tiles(M, 256) * dense_tiles(N, 256), steps = dense_tiles(K_all, 64);
    int best = 1;
    int64_t least = (steps + 8) * 3 / 4;             // the pieces have to be written, read and added up
    for (int s = 2; s <= 32 && tiles < kDensePairs && steps / s >= 8; ++s) {
        const int64_t t = dense_tiles(tiles * s, kDensePairs) * (dense_tiles(steps, s) + 8);
        if (t < least) {
            least = t;
            best = s;
        }
    }
    return best;
}

}  // namespace mxfp4
