// Tensor maps and launches of the 16-bit product (dense_gemm_kernel.cuh).
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>

#include "../../include/mxfp4.h"
#include "dense_gemm.cuh"
#include "dense_gemm_kernel.cuh"
#include "host_common.cuh"
#include "tma_host.cuh"

namespace mxfp4 {

template <int EPI>
static int launch(const DenseMaps2& maps, const DenseParams& p, int sm_count, cudaStream_t st)
{
    const size_t smem = sizeof(DenseSmem<EPI>) + 1024;
    static PerDeviceOnce once;
    static int resident[kMaxDevices] = {};
    const int dev = current_device();
    if (dev < 0) return MXFP4_ERR_CUDA;
    auto kernel = dense_gemm_kernel<EPI>;
    const int rc = once.run(dev, [&] {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) != cudaSuccess)
            return MXFP4_ERR_CUDA;
        // the persistent grid must not exceed what the device holds at once
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(static_cast<unsigned>(sm_count & ~1), 1, 1);
        cfg.blockDim = dim3(kDThreads, 1, 1);
        cfg.dynamicSmemBytes = smem;
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n <= 0) {
            (void)cudaGetLastError();
            n = sm_count / 2;
        }
        resident[dev] = n < sm_count / 2 ? n : sm_count / 2;
        return resident[dev] > 0 ? MXFP4_OK : MXFP4_ERR_CUDA;
    });
    if (rc != MXFP4_OK) return rc;
    const int64_t items = static_cast<int64_t>(p.q[0].items) + p.q[1].items;
    const int clusters = static_cast<int>(items < resident[dev] ? items : resident[dev]);
    return launch_kernel_pdl(kernel, 2 * clusters, kDThreads, smem, st, maps, p) == cudaSuccess ? MXFP4_OK : MXFP4_ERR_CUDA;
}

static bool operand_map(CUtensorMap* map, const DenseMatrix& m, bool mn, int64_t rows, int64_t K, int box_rows = kDHalf)
{
    return mn ? make_tmap_2d(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, m.p, K, rows, m.ld * 2, 64, 64, CU_TENSOR_MAP_SWIZZLE_128B)
              : make_tmap_2d(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, m.p, rows, K, m.ld * 2, box_rows, kDBlockK,
                             CU_TENSOR_MAP_SWIZZLE_128B);
}

// Sizes and tensor maps of one product; `outs` outputs of `out_cols` columns.
static int prepare(DenseShape& q, DenseMaps& maps, const DenseProduct& c, bool gated, int outs, int64_t out_cols, int width = kDHalf)
{
    const int64_t seg_m = dense_tiles(c.M, kDTile), seg_k = dense_tiles(c.K, kDBlockK);
    const int64_t tiles_n = dense_tiles(c.N, gated ? width : 2 * width);
    const int64_t tiles_m = seg_m * (c.stack_m ? 2 : 1), k_steps = seg_k * (c.stack_k ? 2 : 1);
    if (tiles_m * tiles_n * c.splits > 0x1FFFFFFF || k_steps > kDenseMaxK / kDBlockK) return MXFP4_ERR_SHAPE;
    if (c.splits > 1 && dense_split_rows(c.M) * c.splits > 0x7FFFFFFF) return MXFP4_ERR_SHAPE;
    q.M = static_cast<int32_t>(c.M);
    q.N = static_cast<int32_t>(c.N);
    q.K = static_cast<int32_t>(c.K);
    q.seg_tiles_m = static_cast<int32_t>(seg_m);
    q.tiles_m = static_cast<int32_t>(tiles_m);
    q.tiles_n = static_cast<int32_t>(tiles_n);
    q.seg_k_steps = static_cast<int32_t>(seg_k);
    q.k_steps = static_cast<int32_t>(k_steps);
    q.width = width;
    // A panel of one operand stays in L2 while the other passes, whichever order leaves less to be read from memory; where K
    // is so long that no panel fits, the bands are about as wide as the tiles in flight are high.
    const int64_t fits = kDensePanelBytes / (k_steps * kDBlockK * kDTile * 2);
    const int64_t panel = std::max<int64_t>(8, fits);
    const int64_t band_n = std::min(tiles_n, panel), band_m = std::min(tiles_m, panel);
    q.band_m = tiles_m + dense_tiles(tiles_m, band_m) * tiles_n < tiles_n + dense_tiles(tiles_n, band_n) * tiles_m;
    q.band = static_cast<int32_t>(q.band_m ? band_m : band_n);
    q.hints = fits >= 8;
    q.splits = c.splits;
    q.split_rows = static_cast<int32_t>(dense_split_rows(c.M));
    q.items = static_cast<int32_t>(tiles_m * tiles_n * c.splits);
    q.a_mn = c.a_mn;
    q.out = c.kind;
    const bool out32 = c.kind != kDenseBf16;
    const int n_a = c.stack_m || c.stack_k ? 2 : 1, n_b = gated || c.stack_k ? 2 : 1;
    bool ok = true;
    for (int i = 0; i < n_a && ok; ++i) ok = operand_map(&maps.a[i], c.a[i], c.a_mn, c.M, c.K);
    for (int i = 0; i < n_b && ok; ++i) ok = operand_map(&maps.b[i], c.b[i], c.b_mn, c.N, c.K, width);
    for (int i = 0; i < outs && ok; ++i)
        ok = make_tmap_2d(&maps.out[i], out32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, out32 ? 4 : 2,
                          c.out[i].p, c.splits > 1 ? dense_split_rows(c.M) * c.splits : c.M, out_cols,
                          c.out[i].ld * (out32 ? 4 : 2), 32, out32 ? 32 : 64, CU_TENSOR_MAP_SWIZZLE_128B);
    return ok ? MXFP4_OK : MXFP4_ERR_CUDA;
}

int dense_store(const DenseProduct* products, int n, const DenseExtra* extra, int sm_count, cudaStream_t st)
{
    DenseMaps2 maps;
    DenseParams p;
    memset(&maps, 0, sizeof(maps));
    memset(&p, 0, sizeof(p));
    if (extra) p.x = *extra;
    for (int i = 0; i < n; ++i) {
        const int rc = prepare(p.q[i], maps.q[i], products[i], false, products[i].stack_m ? 2 : 1, products[i].N);
        if (rc != MXFP4_OK) return rc;
    }
    return extra ? launch<kDenseScaled>(maps, p, sm_count, st) : launch<kDenseStore>(maps, p, sm_count, st);
}

int dense_fused(DenseEpilogue epilogue, const DenseProduct& product, const DenseExtra& extra, int sm_count, cudaStream_t st)
{
    DenseMaps2 maps;
    DenseParams p;
    memset(&maps, 0, sizeof(maps));
    memset(&p, 0, sizeof(p));
    p.x = extra;
    const bool gated = epilogue == kDenseGated;
    const int outs = epilogue == kDensePartials ? 0 : gated && extra.keep ? 3 : 1;
    const int rc = prepare(p.q[0], maps.q[0], product, gated, outs, epilogue == kDenseLogitGrad ? extra.ld_grad : product.N,
                           epilogue == kDenseLogitGrad ? kDHalf : dense_width(product.M, product.N, gated ? 1 : 2));
    if (rc != MXFP4_OK) return rc;
    if (gated) return launch<kDenseGated>(maps, p, sm_count, st);
    return epilogue == kDensePartials ? launch<kDensePartials>(maps, p, sm_count, st)
                                      : launch<kDenseLogitGrad>(maps, p, sm_count, st);
}

// The sum of a split product's pieces in their order, rounded to bf16.
struct RoundRowsParams {
    const float* from;           // [pieces][rows x cols]
    int64_t piece;               // elements from one piece to the next
    int32_t pieces;
    __nv_bfloat16* to;
    int64_t ld, items;           // items: rows * cols / 8
    int32_t per_row;
};

__global__ void __launch_bounds__(256) round_rows_kernel(const RoundRowsParams p)
{
    griddep_launch_dependents();
    griddep_wait();
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < p.items; i += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t row = i / p.per_row, col = (i - row * p.per_row) * 8;
        float2 v[4] = {};
#pragma unroll 4
        for (int s = 0; s < p.pieces; ++s) {
            const float4* from = reinterpret_cast<const float4*>(p.from + s * p.piece + i * 8);
            const float4 a = from[0], b = from[1];
            v[0] = make_float2(v[0].x + a.x, v[0].y + a.y);
            v[1] = make_float2(v[1].x + a.z, v[1].y + a.w);
            v[2] = make_float2(v[2].x + b.x, v[2].y + b.y);
            v[3] = make_float2(v[3].x + b.z, v[3].y + b.w);
        }
        *reinterpret_cast<uint4*>(p.to + row * p.ld + col) = pack8(v);
    }
}

int dense_round(const float* from, int pieces, int64_t rows, int64_t cols, void* to, int64_t ld, int sm_count, cudaStream_t st)
{
    RoundRowsParams p;
    p.from = from;
    p.piece = dense_split_rows(rows) * cols;
    p.pieces = pieces;
    p.to = static_cast<__nv_bfloat16*>(to);
    p.ld = ld;
    p.items = rows * (cols / 8);
    p.per_row = static_cast<int32_t>(cols / 8);
    const int64_t blocks = (p.items + 255) / 256, most = 8 * static_cast<int64_t>(sm_count);
    return launch_kernel_pdl(round_rows_kernel, static_cast<int>(blocks < most ? blocks : most), 256, 0, st, p) == cudaSuccess
               ? MXFP4_OK : MXFP4_ERR_CUDA;
}

// Status word of this translation unit's kernels, cleared when it is set.
int dense_take_status(int* status) { return take_unit_status(status); }
int dense_selftest(cudaStream_t st) { return unit_selftest(st); }

}  // namespace mxfp4
