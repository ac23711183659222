// The 16-bit product with its fused epilogues as the other translation units call it (see dense_gemm_kernel.cuh).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace mxfp4 {

enum DenseEpilogue { kDenseBf16, kDenseF32, kDenseAddF32, kDenseGated, kDensePartials, kDenseLogitGrad };

constexpr int64_t kDenseMaxDim = 0x7FFFFF00;

// What the kernel reads besides its tensor maps.
struct DenseParams {
    int32_t M, N, K;             // of one segment; gated: N features of each projection
    int32_t tiles_m, tiles_n;    // of all segments
    int32_t seg_tiles_m;
    int32_t k_steps;             // of all segments
    int32_t seg_k_steps;
    int32_t band;                // tile columns per band of the tile order
    // gated
    int32_t act;
    int32_t keep;                // g and u are stored too
    // log probabilities: columns col_base .. col_base + N of `vocab`
    int64_t vocab, col_base;
    const int64_t* targets;
    float scale;
    const float* lse;
    const float* d_logp;
    const float* d_lse;
    float2* parts;               // [ceil(N / 128)][ld_parts]: maximum, sum of exponentials
    int64_t ld_parts;
    float* picked;               // the target's value
    int32_t ld_grad;             // columns of the gradient's buffer, those past N set to 0
};

struct DenseMatrix {
    const void* p;
    int64_t ld;                  // elements
};

// One launch.  a and b are stored along K, or (a_mn, b_mn) along their own rows: [K x M], [K x N].  `stack_m`: two
// matrices a, each with its own output; `stack_k`: two pairs (a, b) whose products are added.
struct DenseCall {
    DenseEpilogue epilogue;
    bool a_mn = false, b_mn = false;
    bool stack_m = false, stack_k = false;
    DenseMatrix a[2] = {}, b[2] = {}, out[3] = {};
    DenseParams p = {};
};

int dense_launch(DenseCall& call, int sm_count, cudaStream_t st);

inline int64_t dense_tiles(int64_t n, int64_t tile) { return (n + tile - 1) / tile; }

}  // namespace mxfp4
