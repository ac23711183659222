// Log probabilities of given tokens from an output layer's input and weight (see include/mxfp4.h).
//
// Forward: the logits' product leaves only a maximum and a sum of exponentials per row and 128 columns, and the target's
// value; a second kernel joins them.  Backward, piece by piece of the vocabulary: the piece's logits again, whose
// epilogue forms their gradient (bf16, in the workspace), then its product with the piece of the weight, added to the
// input's gradient in fp32, and with the input, which is the piece of the weight's gradient.
//
// Bound by the products: 8192 tokens of 4096 features, vocabulary 128256, forward 5430 to 5700 us by itself (1.5 to 1.6 PFLOP/s),
// 6060 to 6600 pass after pass, on one device and another: the power cap sustains 1.3 to 1.42; 19 us are the join.  Backward,
// 4096 tokens: 8320 to 8470, and 9100 to 9970; of 16 and 64 tokens 630 and 660, where a weight read once and its gradient
// take 325: the logits' product and dx each read it.
//
// The gradient of the logits is rounded to bf16 because it is an operand of the tensor cores' products: sums over
// hundreds of them are off by about 0.0017 of their value (norm), as much as the rounding of a bf16 result.  What the
// positions' gradients have in common is not rounded but multiplied into the sums (dense_common): that of a mean over 255
// positions, 1/255, would be 0.0039 off, and all of dx and dW with it.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/mxfp4.h"
#include "dense_gemm.cuh"
#include "host_common.cuh"
#include "row_io.cuh"
#include "ptx_sm100.cuh"
#include "tma_host.cuh"

namespace mxfp4 {

// Rows per forward product: bounds the partial results' memory (131 MB at a vocabulary of 128256) with tens of thousands
// of tiles in a launch.
constexpr int64_t kLossRows = 16384;

struct LossJoinParams {
    const float2* parts;         // [pieces][ld_parts]
    const float* picked;
    const int64_t* targets;
    float* logp;
    float* lse;
    int64_t ld_parts, vocab;
    int32_t rows, pieces;
};

constexpr int kJoinWarps = 32;
constexpr int kJoinUnroll = 4;   // partial results in flight per lane

// 32 rows per CTA, one per lane; the warps take the partial results in turn and are joined in their order.
__global__ void __launch_bounds__(kJoinWarps * 32) loss_join_kernel(const LossJoinParams p)
{
    __shared__ float2 part[kJoinWarps][32];
    griddep_launch_dependents();
    griddep_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int row = blockIdx.x * 32 + lane;
    // sums are relative to the maximum so far; while that is -infinity they are 0
    auto join = [](float2& a, const float2& b) {
        const float m = fmaxf(a.x, b.x), ref = m == -INFINITY ? 0.0f : m;
        a = make_float2(m, a.y * __expf(a.x - ref) + b.y * __expf(b.x - ref));
    };
    float2 v = make_float2(-INFINITY, 0.0f);
    if (row < p.rows) {
        for (int i = warp; i < p.pieces; i += kJoinWarps * kJoinUnroll) {
            float2 w[kJoinUnroll];
#pragma unroll
            for (int u = 0; u < kJoinUnroll; ++u)
                w[u] = i + u * kJoinWarps < p.pieces ? p.parts[(i + u * kJoinWarps) * p.ld_parts + row] : make_float2(-INFINITY, 0.0f);
#pragma unroll
            for (int u = 0; u < kJoinUnroll; ++u) join(v, w[u]);
        }
    }
    smem_store(&part[warp][lane], v, part, sizeof(part));
    __syncthreads();
    if (warp != 0 || row >= p.rows) return;
    for (int w = 1; w < kJoinWarps; ++w) join(v, smem_load<float2>(&part[w][lane], part, sizeof(part)));
    const float total = logf(v.y);
    p.lse[row] = v.x + total;                              // -infinity - infinity where all are masked
    if (!p.logp) return;
    const int64_t t = p.targets[row];
    float logp = 0.0f;
    if (t >= p.vocab) logp = NAN;
    else if (t >= 0) logp = v.y == 0.0f ? -INFINITY : (p.picked[row] - v.x) - total;
    p.logp[row] = logp;
}

// Columns of the vocabulary per piece of the backward pass: 256 MB of gradients, at least 8192 columns, so that the fp32
// sums of dx, which every piece reads and writes once, stay a small part of the traffic.
static int64_t loss_piece(int64_t tokens, int64_t vocab)
{
    int64_t cols = (int64_t{1} << 27) / tokens / 256 * 256;
    if (cols < 8192) cols = 8192;
    return cols < vocab ? cols : vocab;
}

// Partial results per row of a forward product.
static int64_t loss_pieces(int64_t rows, int64_t vocab) { return rows > 0 ? dense_tiles(vocab, dense_width(rows, vocab, 2)) : 0; }

static size_t loss_grad_bytes(int64_t tokens, int64_t vocab)
{
    return round_up(static_cast<size_t>(tokens) * round_up(loss_piece(tokens, vocab), 8) * 2, 256);
}

static int loss_check(const void* x, int64_t ld_x, const void* w, int64_t ld_w, int64_t tokens, int64_t in_features,
                      int64_t vocab, float scale)
{
    if (!x || !w) return MXFP4_ERR_NULL;
    if (!(scale > 0.0f) || isinf(scale)) return MXFP4_ERR_ENUM;
    if (tokens <= 0 || in_features <= 0 || vocab <= 0 || in_features % 8 != 0 || tokens > kDenseMaxDim ||
        in_features > kDenseMaxK || vocab > kDenseMaxDim)
        return MXFP4_ERR_SHAPE;
    if (ld_x < in_features || ld_w < in_features) return MXFP4_ERR_SHAPE;
    if (!aligned16(x) || !aligned16(w) || ld_x % 8 != 0 || ld_w % 8 != 0) return MXFP4_ERR_ALIGN;
    return MXFP4_OK;
}

int linear_logprobs_take_status(int* status) { return take_unit_status(status); }
int linear_logprobs_selftest(cudaStream_t st) { return unit_selftest(st); }

}  // namespace mxfp4

using namespace mxfp4;

extern "C" {

size_t mxfp4_linear_logprobs_workspace_bytes(int64_t tokens, int64_t in_features, int64_t vocab, int backward)
{
    if (tokens <= 0 || in_features <= 0 || vocab <= 0 || in_features % 8 != 0 || in_features > kDenseMaxK ||
        tokens > (backward ? kDenseMaxK : kDenseMaxDim) || vocab > kDenseMaxDim)      // dW sums over the tokens
        return 0;
    if (backward) {
        const int64_t piece = loss_piece(tokens, vocab);
        const int splits = dense_splits(tokens, in_features, piece);
        return loss_grad_bytes(tokens, vocab) +
               (piece == vocab && splits == 1 ? 0 : static_cast<size_t>(splits) * dense_split_rows(tokens) * in_features * 4);
    }
    const size_t rows = round_up(static_cast<size_t>(tokens < kLossRows ? tokens : kLossRows), 32);
    // narrower tiles are for few rows only
    const int64_t pieces = std::max(loss_pieces(std::min(tokens, kLossRows), vocab), loss_pieces(tokens % kLossRows, vocab));
    return rows * static_cast<size_t>(pieces) * sizeof(float2) + rows * sizeof(float);
}

int mxfp4_linear_logprobs_forward(const void* x, int64_t ld_x, const void* w, int64_t ld_w, int64_t tokens,
                                  int64_t in_features, int64_t vocab, const int64_t* targets, float scale, float* logp,
                                  float* lse, void* workspace, size_t workspace_bytes, void* stream)
{
    int rc = loss_check(x, ld_x, w, ld_w, tokens, in_features, vocab, scale);
    if (rc != MXFP4_OK) return rc;
    if (!lse || (targets == nullptr) != (logp == nullptr)) return MXFP4_ERR_NULL;
    const size_t need = mxfp4_linear_logprobs_workspace_bytes(tokens, in_features, vocab, 0);
    if (!workspace || workspace_bytes < need) return MXFP4_ERR_WORKSPACE;
    if (!aligned16(workspace)) return MXFP4_ERR_ALIGN;
    const DeviceInfo& dev = device_info();
    if ((rc = device_status_code(dev)) != MXFP4_OK) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int64_t pitch = round_up(static_cast<size_t>(tokens < kLossRows ? tokens : kLossRows), 32);
    for (int64_t r = 0; r < tokens; r += kLossRows) {
        const int64_t rows = tokens - r < kLossRows ? tokens - r : kLossRows, pieces = loss_pieces(rows, vocab);
        DenseProduct c;
        c.M = rows;
        c.N = vocab;
        c.K = in_features;
        c.a[0] = {static_cast<const __nv_bfloat16*>(x) + r * ld_x, ld_x};
        c.b[0] = {w, ld_w};
        DenseExtra e = {};
        e.vocab = vocab;
        e.targets = targets ? targets + r : nullptr;
        e.scale = scale;
        e.parts = static_cast<float2*>(workspace);
        e.ld_parts = pitch;
        e.picked = reinterpret_cast<float*>(e.parts + pitch * pieces);
        if ((rc = dense_fused(kDensePartials, c, e, dev.sm_count, st)) != MXFP4_OK) return rc;
        LossJoinParams j;
        j.parts = e.parts;
        j.picked = e.picked;
        j.targets = e.targets;
        j.logp = logp ? logp + r : nullptr;
        j.lse = lse + r;
        j.ld_parts = pitch;
        j.vocab = vocab;
        j.rows = static_cast<int32_t>(rows);
        j.pieces = static_cast<int32_t>(pieces);
        if (launch_kernel_pdl(loss_join_kernel, (j.rows + 31) / 32, kJoinWarps * 32, 0, st, j) != cudaSuccess)
            return MXFP4_ERR_CUDA;
    }
    return MXFP4_OK;
}

int mxfp4_linear_logprobs_backward(const void* x, int64_t ld_x, const void* w, int64_t ld_w, int64_t tokens,
                                   int64_t in_features, int64_t vocab, const int64_t* targets, float scale,
                                   const float* lse, const float* d_logp, const float* d_lse, void* dx, int64_t ld_dx,
                                   void* dw, int64_t ld_dw, int dw_dtype, void* workspace, size_t workspace_bytes,
                                   void* stream)
{
    int rc = loss_check(x, ld_x, w, ld_w, tokens, in_features, vocab, scale);
    if (rc != MXFP4_OK) return rc;
    if (!lse || (!d_logp && !d_lse) || (d_logp && !targets) || (!dx && !dw)) return MXFP4_ERR_NULL;
    if (dw_dtype != MXFP4_OUT_BF16 && dw_dtype != MXFP4_OUT_FP32) return MXFP4_ERR_ENUM;
    if (tokens > kDenseMaxK) return MXFP4_ERR_SHAPE;
    if ((dx && ld_dx < in_features) || (dw && ld_dw < in_features)) return MXFP4_ERR_SHAPE;
    if ((dx && (!aligned16(dx) || ld_dx % 8 != 0)) || (dw && (!aligned16(dw) || ld_dw % 8 != 0))) return MXFP4_ERR_ALIGN;
    const size_t need = mxfp4_linear_logprobs_workspace_bytes(tokens, in_features, vocab, 1);
    if (!workspace || workspace_bytes < need) return MXFP4_ERR_WORKSPACE;
    if (!aligned16(workspace)) return MXFP4_ERR_ALIGN;
    const DeviceInfo& dev = device_info();
    if ((rc = device_status_code(dev)) != MXFP4_OK) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);

    const int64_t piece = loss_piece(tokens, vocab);
    const int64_t ld_grad = round_up(piece, 8);
    // the pieces' shares of dx are added up in fp32, those of a split piece side by side
    const int splits = dense_splits(tokens, in_features, piece);
    const bool direct = piece == vocab && splits == 1;
    __nv_bfloat16* grad = static_cast<__nv_bfloat16*>(workspace);
    float* sums = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + loss_grad_bytes(tokens, vocab));
    for (int64_t v = 0; v < vocab; v += piece) {
        const int64_t cols = vocab - v < piece ? vocab - v : piece;
        const DenseMatrix wp = {static_cast<const __nv_bfloat16*>(w) + v * ld_w, ld_w};
        const DenseMatrix gp = {grad, ld_grad};
        DenseProduct c[2];
        c[0].M = tokens;
        c[0].N = cols;
        c[0].K = in_features;
        c[0].a[0] = {x, ld_x};
        c[0].b[0] = wp;
        c[0].out[0] = gp;
        DenseExtra e = {};
        e.vocab = vocab;
        e.col_base = v;
        e.targets = targets;
        e.scale = scale;
        e.lse = lse;
        e.d_logp = d_logp;
        e.d_lse = d_lse;
        e.ld_grad = static_cast<int32_t>(round_up(cols, 8));
        e.rows = static_cast<int32_t>(tokens);
        if ((rc = dense_fused(kDenseLogitGrad, c[0], e, dev.sm_count, st)) != MXFP4_OK) return rc;
        int n = 0;
        if (dx) {
            DenseProduct& q = c[n++] = {};     // dx (+)= dz W
            q.M = tokens;
            q.N = in_features;
            q.K = cols;
            q.b_mn = true;
            q.splits = splits;
            q.kind = direct ? kDenseBf16 : v == 0 ? kDenseF32 : kDenseAddF32;
            q.a[0] = gp;
            q.b[0] = wp;
            q.out[0] = direct ? DenseMatrix{dx, ld_dx} : DenseMatrix{sums, in_features};
        }
        if (dw) {
            DenseProduct& q = c[n++] = {};     // dW = dz^T x
            q.M = cols;
            q.N = in_features;
            q.K = tokens;
            q.a_mn = q.b_mn = true;
            q.kind = dw_dtype == MXFP4_OUT_FP32 ? kDenseF32 : kDenseBf16;
            q.a[0] = gp;
            q.b[0] = {x, ld_x};
            q.out[0] = {static_cast<uint8_t*>(dw) + v * ld_dw * (dw_dtype == MXFP4_OUT_FP32 ? 4 : 2), ld_dw};
        }
        if ((rc = dense_store(c, n, &e, dev.sm_count, st)) != MXFP4_OK) return rc;
    }
    return dx && !direct ? dense_round(sums, splits, tokens, in_features, dx, ld_dx, dev.sm_count, st) : MXFP4_OK;
}

}  // extern "C"
