// Tensor maps and launches of the 16-bit product (dense_gemm_kernel.cuh).
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include "../../include/mxfp4.h"
#include "dense_gemm.cuh"
#include "dense_gemm_kernel.cuh"
#include "host_common.cuh"
#include "tma_host.cuh"

namespace mxfp4 {

template <int EPI, bool A_MN, bool B_MN>
static int launch(const DenseMaps& maps, const DenseParams& p, int sm_count, cudaStream_t st)
{
    const size_t smem = sizeof(DenseSmem) + 1024;
    static PerDeviceOnce once;
    static int resident[kMaxDevices] = {};
    const int dev = current_device();
    if (dev < 0) return MXFP4_ERR_CUDA;
    auto kernel = dense_gemm_kernel<EPI, A_MN, B_MN>;
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
    const int64_t tiles = static_cast<int64_t>(p.tiles_m) * p.tiles_n;
    const int clusters = static_cast<int>(tiles < resident[dev] ? tiles : resident[dev]);
    return launch_kernel_pdl(kernel, 2 * clusters, kDThreads, smem, st, maps, p) == cudaSuccess ? MXFP4_OK : MXFP4_ERR_CUDA;
}

static bool operand_map(CUtensorMap* map, const DenseMatrix& m, bool mn, int64_t rows, int64_t K)
{
    return mn ? make_tmap_2d(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, m.p, K, rows, m.ld * 2, 64, 64, CU_TENSOR_MAP_SWIZZLE_128B)
              : make_tmap_2d(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, m.p, rows, K, m.ld * 2, kDHalf, kDBlockK,
                             CU_TENSOR_MAP_SWIZZLE_128B);
}

int dense_launch(DenseCall& c, int sm_count, cudaStream_t st)
{
    DenseParams& p = c.p;
    const bool gated = c.epilogue == kDenseGated;
    const bool out32 = c.epilogue == kDenseF32 || c.epilogue == kDenseAddF32;
    const int64_t seg_m = dense_tiles(p.M, kDTile), seg_k = dense_tiles(p.K, kDBlockK);
    const int64_t tiles_n = dense_tiles(p.N, gated ? kDHalf : kDTile);
    const int64_t tiles_m = seg_m * (c.stack_m ? 2 : 1), k_steps = seg_k * (c.stack_k ? 2 : 1);
    if (tiles_m * tiles_n > 0x3FFFFFFF || k_steps > 0x3FFFFFFF / kDBlockK) return MXFP4_ERR_SHAPE;
    p.seg_tiles_m = static_cast<int32_t>(seg_m);
    p.tiles_m = static_cast<int32_t>(tiles_m);
    p.tiles_n = static_cast<int32_t>(tiles_n);
    p.seg_k_steps = static_cast<int32_t>(seg_k);
    p.k_steps = static_cast<int32_t>(k_steps);
    p.band = static_cast<int32_t>(tiles_n < 16 ? tiles_n : 16);

    DenseMaps maps;
    memset(&maps, 0, sizeof(maps));
    const int n_a = c.stack_m || c.stack_k ? 2 : 1, n_b = gated || c.stack_k ? 2 : 1;
    for (int i = 0; i < n_a; ++i)
        if (!operand_map(&maps.a[i], c.a[i], c.a_mn, p.M, p.K)) return MXFP4_ERR_CUDA;
    for (int i = 0; i < n_b; ++i)
        if (!operand_map(&maps.b[i], c.b[i], c.b_mn, p.N, p.K)) return MXFP4_ERR_CUDA;
    const int n_out = c.epilogue == kDensePartials ? 0 : gated ? (p.keep ? 3 : 1) : c.stack_m ? 2 : 1;
    for (int i = 0; i < n_out; ++i)
        if (!make_tmap_2d(&maps.out[i], out32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, out32 ? 4 : 2,
                          c.out[i].p, p.M, c.epilogue == kDenseLogitGrad ? p.ld_grad : p.N, c.out[i].ld * (out32 ? 4 : 2), 32,
                          out32 ? 32 : 64, CU_TENSOR_MAP_SWIZZLE_128B))
            return MXFP4_ERR_CUDA;
    switch (c.epilogue) {
        case kDenseGated: return launch<kDenseGated, false, false>(maps, p, sm_count, st);
        case kDensePartials: return launch<kDensePartials, false, false>(maps, p, sm_count, st);
        case kDenseLogitGrad: return launch<kDenseLogitGrad, false, false>(maps, p, sm_count, st);
        case kDenseBf16:
            return c.a_mn ? launch<kDenseBf16, true, true>(maps, p, sm_count, st)
                          : launch<kDenseBf16, false, true>(maps, p, sm_count, st);
        case kDenseF32:
            return c.a_mn ? launch<kDenseF32, true, true>(maps, p, sm_count, st)
                          : launch<kDenseF32, false, true>(maps, p, sm_count, st);
        case kDenseAddF32: return launch<kDenseAddF32, false, true>(maps, p, sm_count, st);
    }
    return MXFP4_ERR_ENUM;
}

// Status word of this translation unit's kernels, cleared when it is set.
int dense_take_status(int* status) { return take_unit_status(status); }

}  // namespace mxfp4
