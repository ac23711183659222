// Host-side construction of TMA tensor maps.  The driver entry point is looked up through
// the runtime so the library links against cudart only.
#pragma once

#include <stdlib.h>

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace mxfp4 {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                  const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn encode_tiled_fn()
{
    // looked up once (initialisation of a function-local static is thread-safe)
    static const EncodeTiledFn fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) !=
                cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            return static_cast<EncodeTiledFn>(nullptr);
        return reinterpret_cast<EncodeTiledFn>(p);
    }();
    return fn;
}

// 2-D row-major tensor [rows x cols] of `elem_bytes`-wide elements with row pitch
// `pitch_bytes`; box = box_cols x box_rows.  Returns false if the driver rejects it.
inline bool make_tmap_2d(CUtensorMap* map, CUtensorMapDataType dtype, uint32_t elem_bytes,
                         const void* base, uint64_t rows, uint64_t cols, uint64_t pitch_bytes,
                         uint32_t box_rows, uint32_t box_cols, CUtensorMapSwizzle swizzle)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {cols, rows};
    cuuint64_t strides[1] = {pitch_bytes};
    cuuint32_t box[2] = {box_cols, box_rows};
    cuuint32_t estr[2] = {1, 1};
    (void)elem_bytes;
    CUresult r = fn(map, dtype, 2, const_cast<void*>(base), dims, strides, box, estr,
                    CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS;
}

// `count` matrices of the 2-D kind, `matrix_bytes` apart: boxes clip at every matrix's own edges.
inline bool make_tmap_3d(CUtensorMap* map, CUtensorMapDataType dtype, const void* base, uint64_t count, uint64_t rows,
                         uint64_t cols, uint64_t pitch_bytes, uint64_t matrix_bytes, uint32_t box_rows,
                         uint32_t box_cols, CUtensorMapSwizzle swizzle)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    cuuint64_t dims[3] = {cols, rows, count};
    cuuint64_t strides[2] = {pitch_bytes, matrix_bytes};
    cuuint32_t box[3] = {box_cols, box_rows, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    CUresult r = fn(map, dtype, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS;
}

// Launch with the programmatic-stream-serialization attribute (see griddep_wait in
// ptx_sm100.cuh).  MXFP4_PDL=0 in the environment turns the attribute off (plain stream order).
inline bool pdl_enabled()
{
    static const bool on = [] {
        const char* e = getenv("MXFP4_PDL");
        return !(e && e[0] == '0');
    }();
    return on;
}

// `cluster` > 1: CTAs come in clusters of that many (for kernels without a compile-time cluster size).
template <typename... KArgs, typename... Args>
inline cudaError_t launch_kernel_pdl_cluster(void (*kernel)(KArgs...), int grid, int block, size_t smem, int cluster,
                                             cudaStream_t stream, Args&&... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(grid), 1, 1);
    cfg.blockDim = dim3(static_cast<unsigned>(block), 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    unsigned n = 0;
    if (pdl_enabled()) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = static_cast<unsigned>(cluster);
        attr[n].val.clusterDim.y = 1;
        attr[n++].val.clusterDim.z = 1;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

template <typename... KArgs, typename... Args>
inline cudaError_t launch_kernel_pdl(void (*kernel)(KArgs...), int grid, int block, size_t smem, cudaStream_t stream,
                                     Args&&... args)
{
    return launch_kernel_pdl_cluster(kernel, grid, block, smem, 1, stream, static_cast<Args&&>(args)...);
}

}  // namespace mxfp4
