// Gated projections of a feed-forward block kept in 16 bits (see include/mxfp4.h): argument checks, the products
// (dense_gemm_kernel.cuh) and the elementwise step of the backward pass.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>

#include "../../include/mxfp4.h"
#include "activations.cuh"
#include "dense_gemm.cuh"
#include "gated_rows_kernel.cuh"
#include "gated_tokens_kernel.cuh"
#include "host_common.cuh"
#include "row_io.cuh"
#include "ptx_sm100.cuh"
#include "tma_host.cuh"

namespace mxfp4 {

// dg = dh * u * act'(g), du = dh * act(g), rounded to bf16: they are operands of the tensor cores' products, whose sums
// over hundreds of them are off by about 0.0017 of their value (norm), as much as the rounding of a bf16 result.
// Eight elements per thread and step, bound by memory: 10 bytes per element (4096 x 14336: 97 us, 6.0 TB/s).
struct GatedGradParams {
    const __nv_bfloat16* dh;
    const __nv_bfloat16* gate;
    const __nv_bfloat16* up;
    __nv_bfloat16* dg;           // [tokens x features]
    __nv_bfloat16* du;
    int64_t ld_dh, ld_kept;
    int64_t items;               // tokens * features / 8
    int32_t per_row;             // features / 8
    int32_t act;
};

constexpr int kGradThreads = 256;

__global__ void __launch_bounds__(kGradThreads) gated_grad_kernel(const GatedGradParams p)
{
    griddep_launch_dependents();
    griddep_wait();
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kGradThreads;
    with_act(p.act, [&](auto act) {
        for (int64_t i = static_cast<int64_t>(blockIdx.x) * kGradThreads + threadIdx.x; i < p.items; i += stride) {
            const int64_t row = i / p.per_row;
            const int64_t col = (i - row * p.per_row) * 8;
            float2 dh[4], g[4], u[4], a[4], b[4];
            const uint4 w0 = ld_stream(p.dh + row * p.ld_dh + col);
            const uint4 w1 = ld_stream(p.gate + row * p.ld_kept + col);
            const uint4 w2 = ld_stream(p.up + row * p.ld_kept + col);
            unpack8(w0, dh);
            unpack8(w1, g);
            unpack8(w2, u);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 x = act_both<decltype(act)::value>(g[j].x), y = act_both<decltype(act)::value>(g[j].y);
                a[j] = make_float2(dh[j].x * u[j].x * x.y, dh[j].y * u[j].y * y.y);
                b[j] = make_float2(dh[j].x * x.x, dh[j].y * y.x);
            }
            *reinterpret_cast<uint4*>(p.dg + i * 8) = pack8(a);
            *reinterpret_cast<uint4*>(p.du + i * 8) = pack8(b);
        }
    });
}

// Whether the kernel with the weights as rows takes a forward pass: up to 160 tokens, where it computes for fewer rows than the
// tile of 256 that the other one computes for in any case, and beyond that where its tiles, which need only be a multiple of 16
// tokens, hold at most 7/8 of the other's rows and K is long enough for its epilogue.  4096 x 14336, pass after pass on one
// device, this kernel and the other: 16 tokens 41 and 48 us, 64 42 and 49, 128 47 and 51, 160 49 and 52, 200 55 and 53, 240 58
// and 54, 333 78 and 87, 400 86 and 89, 512 97 and 93, 600 111 and 123, 1100 180 and 196; of 600 tokens with other
// weights: 4096 x 2048 34 and 30, 4096 x 8192 70 and 76, 4096 x 28672 216 and 253, 2048 x 8192 43 and 45, 1024 x 4096 24 and 19.
static bool gated_as_columns(int64_t tokens, int64_t in_features)
{
    const int64_t tiles = dense_tiles(tokens, 256), rows = tiles * dense_tiles(dense_tiles(tokens, tiles), 16) * 16;
    return tokens <= 160 || (in_features >= 2048 && tokens > 256 && rows * 8 <= tiles * 256 * 7);
}

static int gated_tokens(const mxfp4_gated_desc& d, void* h, int64_t ld_h, void* gate, void* up, int64_t ld_kept, int sm_count,
                        cudaStream_t st)
{
    const size_t smem = sizeof(GatedTokensSmem) + 1024;
    static PerDeviceOnce once;
    static int resident[kMaxDevices] = {};
    const int dev = current_device();
    if (dev < 0) return MXFP4_ERR_CUDA;
    const int rc = once.run(dev, [&] {
        if (cudaFuncSetAttribute(gated_tokens_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) !=
            cudaSuccess)
            return MXFP4_ERR_CUDA;
        // the persistent grid must not exceed what the device holds at once
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(static_cast<unsigned>(sm_count & ~1), 1, 1);
        cfg.blockDim = dim3(kTThreads, 1, 1);
        cfg.dynamicSmemBytes = smem;
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, gated_tokens_kernel, &cfg) != cudaSuccess || n <= 0) {
            (void)cudaGetLastError();
            n = sm_count / 2;
        }
        resident[dev] = n < sm_count / 2 ? n : sm_count / 2;
        return resident[dev] > 0 ? MXFP4_OK : MXFP4_ERR_CUDA;
    });
    if (rc != MXFP4_OK) return rc;
    const int64_t tiles_n = dense_tiles(d.tokens, 256), tile_tokens = dense_tiles(dense_tiles(d.tokens, tiles_n), 16) * 16;
    GatedTokensMaps maps;
    memset(&maps, 0, sizeof(maps));
    const auto bf16 = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    const auto swizzle = CU_TENSOR_MAP_SWIZZLE_128B;
    void* outs[3] = {h, gate, up};
    bool ok = make_tmap_2d(&maps.w[0], bf16, 2, d.w_gate, d.features, d.in_features, d.ld_gate * 2, 64, kTBlockK, swizzle) &&
              make_tmap_2d(&maps.w[1], bf16, 2, d.w_up, d.features, d.in_features, d.ld_up * 2, 64, kTBlockK, swizzle) &&
              make_tmap_2d(&maps.x, bf16, 2, d.x, d.tokens, d.in_features, d.ld_x * 2, static_cast<uint32_t>(tile_tokens / 2),
                           kTBlockK, swizzle);
    for (int i = 0; i < (gate ? 3 : 1) && ok; ++i)
        ok = make_tmap_2d(&maps.out[i], bf16, 2, outs[i], d.tokens, d.features, (i ? ld_kept : ld_h) * 2, kTBox, 64, swizzle);
    if (!ok) return MXFP4_ERR_CUDA;
    GatedTokensParams p;
    p.tokens = static_cast<int32_t>(d.tokens);
    p.features = static_cast<int32_t>(d.features);
    p.K = static_cast<int32_t>(d.in_features);
    p.tile_tokens = static_cast<int32_t>(tile_tokens);
    p.tiles_n = static_cast<int32_t>(tiles_n);
    p.tiles = static_cast<int32_t>(tiles_n * dense_tiles(d.features, kTFeatures));
    p.k_steps = static_cast<int32_t>(dense_tiles(d.in_features, kTBlockK));
    p.stage_bytes = kTWeightBytes + p.tile_tokens / 2 * 128;
    p.stages = std::min(kTMostStages, kTRing / p.stage_bytes);
    p.act = d.act;
    p.keep = gate != nullptr;
    const int clusters = p.tiles < resident[dev] ? p.tiles : resident[dev];
    return launch_kernel_pdl(gated_tokens_kernel, 2 * clusters, kTThreads, smem, st, maps, p) == cudaSuccess ? MXFP4_OK
                                                                                                           : MXFP4_ERR_CUDA;
}

int gated_linear_take_status(int* status) { return take_unit_status(status); }
int gated_linear_selftest(cudaStream_t st) { return unit_selftest(st); }

static size_t gated_grad_bytes(int64_t tokens, int64_t features)
{
    return round_up(static_cast<size_t>(tokens) * features * 2, 256);
}

// Whether the backward pass takes these sizes: sums go over the features of both projections (dx) and over the tokens (dW).
static bool gated_backward_takes(int64_t tokens, int64_t in_features, int64_t features)
{
    return tokens <= kDenseMaxK && in_features <= kDenseMaxK && features <= kDenseMaxK / 2 / 64 * 64;
}

// Sizes, leading dimensions and alignment of what both directions read.
static int gated_check(const mxfp4_gated_desc* d)
{
    if (!d || !d->x || !d->w_gate || !d->w_up) return MXFP4_ERR_NULL;
    if (d->act < MXFP4_GATE_LINEAR || d->act > MXFP4_GATE_RELU) return MXFP4_ERR_ENUM;
    if (d->tokens <= 0 || d->in_features <= 0 || d->features <= 0 || d->in_features % 8 != 0 || d->features % 8 != 0)
        return MXFP4_ERR_SHAPE;
    if (d->tokens > kDenseMaxDim || d->in_features > kDenseMaxK || d->features > kDenseMaxDim) return MXFP4_ERR_SHAPE;
    if (d->ld_x < d->in_features || d->ld_gate < d->in_features || d->ld_up < d->in_features) return MXFP4_ERR_SHAPE;
    if (!aligned16(d->x) || !aligned16(d->w_gate) || !aligned16(d->w_up) || d->ld_x % 8 != 0 || d->ld_gate % 8 != 0 ||
        d->ld_up % 8 != 0)
        return MXFP4_ERR_ALIGN;
    return MXFP4_OK;
}

}  // namespace mxfp4

using namespace mxfp4;

extern "C" {

int mxfp4_gated_linear_forward(const mxfp4_gated_desc* d, void* h, int64_t ld_h, void* gate, void* up, int64_t ld_kept,
                               void* stream)
{
    int rc = gated_check(d);
    if (rc != MXFP4_OK) return rc;
    if (!h || (gate == nullptr) != (up == nullptr)) return MXFP4_ERR_NULL;
    if (ld_h < d->features || (gate && ld_kept < d->features)) return MXFP4_ERR_SHAPE;
    if (!aligned16(h) || ld_h % 8 != 0 || (gate && (!aligned16(gate) || !aligned16(up) || ld_kept % 8 != 0)))
        return MXFP4_ERR_ALIGN;
    const DeviceInfo& dev = device_info();
    if ((rc = device_status_code(dev)) != MXFP4_OK) return rc;
    if (d->tokens <= kGRowsTokens) {
        GatedRowsParams p;
        p.x = static_cast<const __nv_bfloat16*>(d->x);
        p.w_gate = static_cast<const __nv_bfloat16*>(d->w_gate);
        p.w_up = static_cast<const __nv_bfloat16*>(d->w_up);
        p.h = static_cast<__nv_bfloat16*>(h);
        p.gate = static_cast<__nv_bfloat16*>(gate);
        p.up = static_cast<__nv_bfloat16*>(up);
        p.ld_x = d->ld_x;
        p.ld_gate = d->ld_gate;
        p.ld_up = d->ld_up;
        p.ld_h = ld_h;
        p.ld_kept = ld_kept;
        p.tokens = static_cast<int32_t>(d->tokens);
        p.features = static_cast<int32_t>(d->features);
        p.K = static_cast<int32_t>(d->in_features);
        p.act = d->act;
        return launch_kernel_pdl(gated_rows_kernel, static_cast<int>(d->features / kGRowsFeatures), kGRowsWarps * 32, 0,
                                 static_cast<cudaStream_t>(stream), p) == cudaSuccess
                   ? MXFP4_OK : MXFP4_ERR_CUDA;
    }
    if (gated_as_columns(d->tokens, d->in_features))
        return gated_tokens(*d, h, ld_h, gate, up, ld_kept, dev.sm_count, static_cast<cudaStream_t>(stream));
    DenseProduct c;
    c.M = d->tokens;
    c.N = d->features;
    c.K = d->in_features;
    c.a[0] = {d->x, d->ld_x};
    c.b[0] = {d->w_gate, d->ld_gate};
    c.b[1] = {d->w_up, d->ld_up};
    c.out[0] = {h, ld_h};
    c.out[1] = {gate, ld_kept};
    c.out[2] = {up, ld_kept};
    DenseExtra extra = {};
    extra.act = d->act;
    extra.keep = gate != nullptr;
    for (int i = 0; i < 3; ++i) {
        extra.out[i] = static_cast<__nv_bfloat16*>(const_cast<void*>(c.out[i].p));
        extra.ld_out[i] = c.out[i].ld;
    }
    return dense_fused(kDenseGated, c, extra, dev.sm_count, static_cast<cudaStream_t>(stream));
}

size_t mxfp4_gated_linear_workspace_bytes(int64_t tokens, int64_t in_features, int64_t features)
{
    if (tokens <= 0 || in_features <= 0 || features <= 0 || in_features % 8 != 0 || features % 8 != 0 ||
        !gated_backward_takes(tokens, in_features, features))
        return 0;
    const int splits = dense_splits(tokens, in_features, 2 * features);
    return 2 * gated_grad_bytes(tokens, features) +
           (splits > 1 ? static_cast<size_t>(splits) * dense_split_rows(tokens) * in_features * 4 : 0);
}

int mxfp4_gated_linear_backward(const mxfp4_gated_desc* d, const void* dh, int64_t ld_dh, const void* gate, const void* up,
                                int64_t ld_kept, void* dx, int64_t ld_dx, void* dw_gate, void* dw_up, int64_t ld_dw,
                                int dw_dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    int rc = gated_check(d);
    if (rc != MXFP4_OK) return rc;
    if (!dh || !gate || !up || (dw_gate == nullptr) != (dw_up == nullptr) || (!dx && !dw_gate)) return MXFP4_ERR_NULL;
    if (dw_dtype != MXFP4_OUT_BF16 && dw_dtype != MXFP4_OUT_FP32) return MXFP4_ERR_ENUM;
    if (!gated_backward_takes(d->tokens, d->in_features, d->features)) return MXFP4_ERR_SHAPE;
    if (ld_dh < d->features || ld_kept < d->features || (dx && ld_dx < d->in_features) || (dw_gate && ld_dw < d->in_features))
        return MXFP4_ERR_SHAPE;
    if (!aligned16(dh) || !aligned16(gate) || !aligned16(up) || ld_dh % 8 != 0 || ld_kept % 8 != 0 ||
        (dx && (!aligned16(dx) || ld_dx % 8 != 0)) || (dw_gate && (!aligned16(dw_gate) || !aligned16(dw_up) || ld_dw % 8 != 0)))
        return MXFP4_ERR_ALIGN;
    const size_t need = mxfp4_gated_linear_workspace_bytes(d->tokens, d->in_features, d->features);
    if (!workspace || workspace_bytes < need) return MXFP4_ERR_WORKSPACE;
    if (!aligned16(workspace)) return MXFP4_ERR_ALIGN;
    const DeviceInfo& dev = device_info();
    if ((rc = device_status_code(dev)) != MXFP4_OK) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);

    GatedGradParams g;
    g.dh = static_cast<const __nv_bfloat16*>(dh);
    g.gate = static_cast<const __nv_bfloat16*>(gate);
    g.up = static_cast<const __nv_bfloat16*>(up);
    g.dg = static_cast<__nv_bfloat16*>(workspace);
    g.du = reinterpret_cast<__nv_bfloat16*>(static_cast<uint8_t*>(workspace) + gated_grad_bytes(d->tokens, d->features));
    g.ld_dh = ld_dh;
    g.ld_kept = ld_kept;
    g.items = d->tokens * (d->features / 8);
    g.per_row = static_cast<int32_t>(d->features / 8);
    g.act = d->act;
    const int64_t blocks = (g.items + kGradThreads - 1) / kGradThreads;
    const int64_t most = 8 * static_cast<int64_t>(dev.sm_count);
    if (launch_kernel_pdl(gated_grad_kernel, static_cast<int>(blocks < most ? blocks : most), kGradThreads, 0, st, g) !=
        cudaSuccess)
        return MXFP4_ERR_CUDA;
    const DenseMatrix mg = {g.dg, d->features}, mu = {g.du, d->features};
    DenseProduct c[2];
    int n = 0;
    const int splits = dense_splits(d->tokens, d->in_features, 2 * d->features);
    float* sums = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + 2 * gated_grad_bytes(d->tokens, d->features));
    if (dx) {
        DenseProduct& x = c[n++];          // dx = dg Wg + du Wu
        x.M = d->tokens;
        x.N = d->in_features;
        x.K = d->features;
        x.b_mn = x.stack_k = true;
        x.splits = splits;
        x.kind = splits > 1 ? kDenseF32 : kDenseBf16;
        x.a[0] = mg;
        x.a[1] = mu;
        x.b[0] = {d->w_gate, d->ld_gate};
        x.b[1] = {d->w_up, d->ld_up};
        x.out[0] = splits > 1 ? DenseMatrix{sums, d->in_features} : DenseMatrix{dx, ld_dx};
    }
    if (dw_gate) {
        DenseProduct& w = c[n++];          // dWg = dg^T x, dWu = du^T x
        w.M = d->features;
        w.N = d->in_features;
        w.K = d->tokens;
        w.a_mn = w.b_mn = w.stack_m = true;
        w.kind = dw_dtype == MXFP4_OUT_FP32 ? kDenseF32 : kDenseBf16;
        w.a[0] = mg;
        w.a[1] = mu;
        w.b[0] = {d->x, d->ld_x};
        w.out[0] = {dw_gate, ld_dw};
        w.out[1] = {dw_up, ld_dw};
    }
    if ((rc = dense_store(c, n, nullptr, dev.sm_count, st)) != MXFP4_OK || !dx || splits == 1) return rc;
    return dense_round(sums, splits, d->tokens, d->in_features, dx, ld_dx, dev.sm_count, st);
}

}  // extern "C"
