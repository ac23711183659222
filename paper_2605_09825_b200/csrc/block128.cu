// C ABI of the 8-bit product with one fp32 scale per 128 elements (see include/mxfp4.h): argument
// checks, tensor maps and launches.
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include "../../include/mxfp4.h"
#include "host_common.cuh"
#include "ptx_sm100.cuh"
#include "tma_host.cuh"
#include "block128_quantize_kernel.cuh"
#include "block128_gemm_kernel.cuh"
#include "block128_rows_kernel.cuh"

namespace mxfp4 {

// Output tiles are spread over the pairs of this many SMs when a product is split along K; a constant
// so that the workspace size needs no device.
constexpr int kB128SplitPairs = 74;

static int64_t blocks_of(int64_t n) { return (n + kB128 - 1) / kB128; }

static Quant128Params quantize128_params(const void* src, int64_t rows, int64_t cols, int64_t ld, int axis, bool square,
                                         void* codes, void* scales)
{
    Quant128Params p;
    p.src = static_cast<const __nv_bfloat16*>(src);
    p.codes = static_cast<uint8_t*>(codes);
    p.scales = static_cast<float*>(scales);
    p.ld = ld;
    p.rows = static_cast<int32_t>(rows);
    p.cols = static_cast<int32_t>(cols);
    p.tiles_c = static_cast<int32_t>(blocks_of(cols));
    const int64_t outer = axis == MXFP4_AXIS_COLS ? rows : cols;
    p.pitch = static_cast<int32_t>(square ? blocks_of(outer) : blocks_of(outer) * kB128);
    return p;
}

static int64_t quantize128_tiles(int64_t rows, int64_t cols) { return blocks_of(rows) * blocks_of(cols); }

static int64_t gemm128_tiles(int64_t M, int64_t N) { return ((M + kBTile - 1) / kBTile) * ((N + kBTile - 1) / kBTile); }

// Up to this many rows of A the product is bound by reading B and runs without the tensor cores' machinery
// (1 x 4096 x 14336: 13.4 us against 22 + 5 us of the split kernel and its join).
static bool gemm128_few_rows(int64_t M) { return M <= 8 * kRowsMaxTiles; }

// Which tiles are split along K, and into how many pieces: those that do not fill a wave of the pairs, into as
// many pieces as fit the wave, with at least four K-steps in each -- where that makes the wave at least 12 K-steps
// shorter, which is what the second kernel and the traffic of the sums cost: 4096 x 4096 x 2048 in two pieces (8
// K-steps less) 44 us, whole 41 us; 333 x 28672 x 1024 (4 less) 26 and 24 us; 4096 x 4096 x 4096 with a
// scale per row (16 less) 93.5 and 95.6 us; 333 x 28672 x 4096 (28 less) 71 and 84 us.
struct Split128 {
    int64_t whole;               // tiles of one piece
    int64_t split;               // tiles after them
    int64_t pieces;              // of each of these
};

static Split128 gemm128_split(int64_t M, int64_t N, int64_t K)
{
    const int64_t tiles = gemm128_tiles(M, N), steps = blocks_of(K);
    const int64_t left = tiles % kB128SplitPairs;
    int64_t pieces = left > 0 ? kB128SplitPairs / left : 1;
    if (pieces > steps / 4) pieces = steps / 4;
    if (gemm128_few_rows(M) || pieces < 2 || steps - steps / pieces < 12) return {tiles, 0, 1};
    return {tiles - left, left, pieces};
}

static int gemm128_shape_ok(int64_t M, int64_t N, int64_t K)
{
    if (M <= 0 || N <= 0 || K <= 0 || K % 16 != 0) return MXFP4_ERR_SHAPE;
    if (M > 0x7FFFFF00 || N > 0x7FFFFF00 || K > 0x7FFFFF00) return MXFP4_ERR_SHAPE;
    const int64_t tiles = gemm128_tiles(M, N);
    return tiles <= 0x7FFFFFFF / blocks_of(K) && tiles <= 0x3FFFFFFF ? MXFP4_OK : MXFP4_ERR_SHAPE;
}

template <bool BROWS, bool OUT32>
static int launch_gemm128(const CUtensorMap& tm_a, const CUtensorMap& tm_b, const CUtensorMap& tm_out,
                          const CUtensorMap& tm_parts, const Gemm128Params& p, int sm_count, cudaStream_t st)
{
    const size_t smem = sizeof(Gemm128Smem) + 1024;
    static PerDeviceOnce once;
    static int resident[kMaxDevices] = {};
    const int dev = current_device();
    if (dev < 0) return MXFP4_ERR_CUDA;
    auto kernel = gemm_block128_pair_kernel<BROWS, OUT32>;
    const int rc = once.run(dev, [&] {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) !=
            cudaSuccess)
            return MXFP4_ERR_CUDA;
        // the persistent grid must not exceed what the device holds at once
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(static_cast<unsigned>(sm_count & ~1), 1, 1);
        cfg.blockDim = dim3(kBThreads, 1, 1);
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
    const int clusters = p.items < resident[dev] ? p.items : resident[dev];
    return launch_kernel_pdl(kernel, 2 * clusters, kBThreads, smem, st, tm_a, tm_b, tm_out, tm_parts, p) ==
                   cudaSuccess
               ? MXFP4_OK : MXFP4_ERR_CUDA;
}

template <bool BROWS, int TILES>
static int launch_rows128(const Rows128Params& p, cudaStream_t st)
{
    const int grid = (p.N + kRowsB - 1) / kRowsB;
    return launch_kernel_pdl(gemm_block128_rows_kernel<BROWS, TILES>, grid, kRowsWarps * 32, 0, st, p) == cudaSuccess
               ? MXFP4_OK : MXFP4_ERR_CUDA;
}

static int rows128_launch(const void* a_codes, const void* a_scales, const void* b_codes, const void* b_scales, bool brows,
                          int64_t M, int64_t N, int64_t K, void* out, int out_dtype, int64_t ld_out, cudaStream_t st)
{
    Rows128Params p;
    p.a_codes = static_cast<const uint8_t*>(a_codes);
    p.b_codes = static_cast<const uint8_t*>(b_codes);
    p.a_scales = static_cast<const float*>(a_scales);
    p.b_scales = static_cast<const float*>(b_scales);
    p.out = out;
    p.ld_out = ld_out;
    p.pitch_a = blocks_of(M) * kB128;
    p.pitch_b = brows ? blocks_of(N) * kB128 : blocks_of(N);
    p.M = static_cast<int32_t>(M);
    p.N = static_cast<int32_t>(N);
    p.K = static_cast<int32_t>(K);
    p.k_blocks = static_cast<int32_t>(blocks_of(K));
    p.out_fp32 = out_dtype == MXFP4_OUT_FP32;
    if (M <= 8) return brows ? launch_rows128<true, 1>(p, st) : launch_rows128<false, 1>(p, st);
    return brows ? launch_rows128<true, 2>(p, st) : launch_rows128<false, 2>(p, st);
}

static int gemm128_launch(const void* a_codes, const void* a_scales, const void* b_codes, const void* b_scales,
                          bool brows, int64_t M, int64_t N, int64_t K, void* out, int out_dtype, int64_t ld_out,
                          void* workspace, int sm_count, cudaStream_t st)
{
    if (gemm128_few_rows(M))
        return rows128_launch(a_codes, a_scales, b_codes, b_scales, brows, M, N, K, out, out_dtype, ld_out, st);
    const Split128 split = gemm128_split(M, N, K);
    const bool out32 = out_dtype == MXFP4_OUT_FP32;
    const int64_t part_rows = M < kBTile ? M : kBTile;
    const int64_t esz = out32 ? 4 : 2;
    const int64_t n_tma = N & ~static_cast<int64_t>(out32 ? 3 : 7);
    CUtensorMap tm_a, tm_b, tm_out, tm_parts;
    memset(&tm_out, 0, sizeof(tm_out));
    memset(&tm_parts, 0, sizeof(tm_parts));
    if (split.whole > 0 && n_tma > 0 &&
        !make_tmap_3d(&tm_out, out32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, out, 1, M, n_tma,
                      ld_out * esz, M * ld_out * esz, 32, out32 ? 32 : 64, CU_TENSOR_MAP_SWIZZLE_128B))
        return MXFP4_ERR_CUDA;
    if (split.split > 0 &&
        !make_tmap_3d(&tm_parts, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, workspace, split.split * split.pieces, part_rows,
                      kBTile, kBTile * 4, part_rows * kBTile * 4, 32, 32, CU_TENSOR_MAP_SWIZZLE_128B))
        return MXFP4_ERR_CUDA;
    if (!make_tmap_2d(&tm_a, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, a_codes, M, K, K, kBHalf, kBBlockK,
                      CU_TENSOR_MAP_SWIZZLE_128B) ||
        !make_tmap_2d(&tm_b, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, b_codes, N, K, K, kBHalf / 2, kBBlockK,
                      CU_TENSOR_MAP_SWIZZLE_128B))
        return MXFP4_ERR_CUDA;
    Gemm128Params p;
    p.a_scales = static_cast<const float*>(a_scales);
    p.b_scales = static_cast<const float*>(b_scales);
    p.out = out;
    p.ld_out = ld_out;
    p.pitch_a = blocks_of(M) * kB128;
    p.pitch_b = brows ? blocks_of(N) * kB128 : blocks_of(N);
    p.M = static_cast<int32_t>(M);
    p.N = static_cast<int32_t>(N);
    p.K = static_cast<int32_t>(K);
    p.tiles_m = static_cast<int32_t>((M + kBTile - 1) / kBTile);
    p.tiles_n = static_cast<int32_t>((N + kBTile - 1) / kBTile);
    int64_t band = (32ll << 20) / (kBTile * K);          // 32 MB of B: a quarter of L2
    if (band < 1) band = 1;
    p.band = static_cast<int32_t>(band < p.tiles_n ? band : p.tiles_n);
    p.k_steps = static_cast<int32_t>(blocks_of(K));
    p.whole = static_cast<int32_t>(split.whole);
    p.splits = static_cast<int32_t>(split.pieces);
    p.items = static_cast<int32_t>(split.whole + split.split * split.pieces);
    p.n_tma = static_cast<int32_t>(n_tma);
    int rc;
    if (brows)
        rc = out32 ? launch_gemm128<true, true>(tm_a, tm_b, tm_out, tm_parts, p, sm_count, st)
                   : launch_gemm128<true, false>(tm_a, tm_b, tm_out, tm_parts, p, sm_count, st);
    else
        rc = out32 ? launch_gemm128<false, true>(tm_a, tm_b, tm_out, tm_parts, p, sm_count, st)
                   : launch_gemm128<false, false>(tm_a, tm_b, tm_out, tm_parts, p, sm_count, st);
    if (rc != MXFP4_OK || split.split == 0) return rc;
    Gemm128JoinParams j;
    j.parts = static_cast<const float*>(workspace);
    j.out = out;
    j.ld_out = ld_out;
    j.M = p.M;
    j.N = p.N;
    j.whole = p.whole;
    j.splits = p.splits;
    j.rows = static_cast<int32_t>(part_rows);
    j.band = p.band;
    j.tiles_m = p.tiles_m;
    j.tiles_n = p.tiles_n;
    j.out_fp32 = out32;
    const int blocks = static_cast<int>(split.split * ((part_rows + kBJoinRows - 1) / kBJoinRows));
    return launch_kernel_pdl(gemm_block128_join_kernel, blocks, 256, 0, st, j) == cudaSuccess ? MXFP4_OK : MXFP4_ERR_CUDA;
}

// (rows, cols, axis) of the pass's operands in their own row-major shapes, and the product's sizes
struct Pass128 {
    int64_t M, N, K;
    int64_t ar, ac, br, bc;
    int a_axis, b_axis, b_shape;
};

static Pass128 pass128(int pass, int64_t T, int64_t in_f, int64_t out_f)
{
    if (pass == MXFP4_PASS_FPROP)
        return {T, out_f, in_f, T, in_f, out_f, in_f, MXFP4_AXIS_COLS, MXFP4_AXIS_COLS, MXFP4_BLOCK_128X128};
    if (pass == MXFP4_PASS_DGRAD)
        return {T, in_f, out_f, T, out_f, out_f, in_f, MXFP4_AXIS_COLS, MXFP4_AXIS_ROWS, MXFP4_BLOCK_128X128};
    return {out_f, in_f, T, T, out_f, T, in_f, MXFP4_AXIS_ROWS, MXFP4_AXIS_ROWS, MXFP4_BLOCK_1X128};
}

// Status word of this translation unit's kernels, cleared when it is set.
int block128_take_status(int* status) { return take_unit_status(status); }

}  // namespace mxfp4

using namespace mxfp4;

extern "C" {

size_t mxfp4_block128_scales_bytes(int64_t outer, int64_t K, int block_shape)
{
    if (outer <= 0 || K <= 0 || K % 16 != 0) return 0;
    const size_t blocks = static_cast<size_t>(blocks_of(outer)) * static_cast<size_t>(blocks_of(K)) * sizeof(float);
    if (block_shape == MXFP4_BLOCK_1X128) return blocks * kB128;
    return block_shape == MXFP4_BLOCK_128X128 ? blocks : 0;
}

int mxfp4_quantize_block128(const void* src_bf16, int64_t rows, int64_t cols, int64_t ld_src, int axis,
                            int block_shape, void* codes, void* scales, void* stream)
{
    if (!src_bf16 || !codes || !scales) return MXFP4_ERR_NULL;
    if (axis != MXFP4_AXIS_ROWS && axis != MXFP4_AXIS_COLS) return MXFP4_ERR_ENUM;
    if (block_shape != MXFP4_BLOCK_1X128 && block_shape != MXFP4_BLOCK_128X128) return MXFP4_ERR_ENUM;
    if (rows <= 0 || cols <= 0 || ld_src < cols) return MXFP4_ERR_SHAPE;
    if ((axis == MXFP4_AXIS_COLS ? cols : rows) % 16 != 0) return MXFP4_ERR_SHAPE;
    if (rows > 0x7FFFFF00 || cols > 0x7FFFFF00 || quantize128_tiles(rows, cols) > 0x3FFFFFFF) return MXFP4_ERR_SHAPE;
    if (!aligned16(src_bf16) || !aligned16(codes) || !aligned16(scales) || ld_src % 8 != 0) return MXFP4_ERR_ALIGN;
    const int rc = device_status_code(device_info());
    if (rc != MXFP4_OK) return rc;
    const bool square = block_shape == MXFP4_BLOCK_128X128;
    const Quant128Params p = quantize128_params(src_bf16, rows, cols, ld_src, axis, square, codes, scales);
    const int grid = static_cast<int>(quantize128_tiles(rows, cols));
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    auto kernel = axis == MXFP4_AXIS_COLS
                      ? (square ? quantize_block128_kernel<1, true> : quantize_block128_kernel<1, false>)
                      : (square ? quantize_block128_kernel<0, true> : quantize_block128_kernel<0, false>);
    return launch_kernel_pdl(kernel, grid, kB128Threads, 0, st, p) == cudaSuccess ? MXFP4_OK : MXFP4_ERR_CUDA;
}

size_t mxfp4_gemm_block128_workspace_bytes(int64_t M, int64_t N, int64_t K)
{
    if (gemm128_shape_ok(M, N, K) != MXFP4_OK) return 0;
    const Split128 split = gemm128_split(M, N, K);
    return static_cast<size_t>(split.split * split.pieces) * (M < kBTile ? M : kBTile) * kBTile * sizeof(float);
}

int mxfp4_gemm_block128(const void* a_codes, const void* a_scales, const void* b_codes, const void* b_scales,
                        int b_block_shape, int64_t M, int64_t N, int64_t K, void* out, int out_dtype, int64_t ld_out,
                        void* workspace, size_t workspace_bytes, void* stream)
{
    if (!a_codes || !a_scales || !b_codes || !b_scales || !out) return MXFP4_ERR_NULL;
    if (out_dtype != MXFP4_OUT_BF16 && out_dtype != MXFP4_OUT_FP32) return MXFP4_ERR_ENUM;
    if (b_block_shape != MXFP4_BLOCK_1X128 && b_block_shape != MXFP4_BLOCK_128X128) return MXFP4_ERR_ENUM;
    int rc = gemm128_shape_ok(M, N, K);
    if (rc != MXFP4_OK) return rc;
    if (ld_out < N) return MXFP4_ERR_SHAPE;
    if (!aligned16(a_codes) || !aligned16(a_scales) || !aligned16(b_codes) || !aligned16(b_scales) || !aligned16(out))
        return MXFP4_ERR_ALIGN;
    if ((ld_out * (out_dtype == MXFP4_OUT_BF16 ? 2 : 4)) % 16 != 0) return MXFP4_ERR_ALIGN;
    const size_t need = mxfp4_gemm_block128_workspace_bytes(M, N, K);
    if (need > 0 && (!workspace || workspace_bytes < need)) return MXFP4_ERR_WORKSPACE;
    if (need > 0 && !aligned16(workspace)) return MXFP4_ERR_ALIGN;
    const DeviceInfo& dev = device_info();
    if ((rc = device_status_code(dev)) != MXFP4_OK) return rc;
    return gemm128_launch(a_codes, a_scales, b_codes, b_scales, b_block_shape == MXFP4_BLOCK_1X128, M, N, K, out,
                          out_dtype, ld_out, workspace, dev.sm_count, static_cast<cudaStream_t>(stream));
}

size_t mxfp4_linear_pass_block128_workspace_bytes(int64_t T, int64_t in_features, int64_t out_features, int pass)
{
    if (pass < 0 || pass > 2 || T <= 0 || in_features <= 0 || out_features <= 0) return 0;
    const Pass128 q = pass128(pass, T, in_features, out_features);
    if (gemm128_shape_ok(q.M, q.N, q.K) != MXFP4_OK) return 0;
    return round_up(static_cast<size_t>(q.M) * q.K, 256) +
           round_up(mxfp4_block128_scales_bytes(q.M, q.K, MXFP4_BLOCK_1X128), 256) +
           round_up(static_cast<size_t>(q.N) * q.K, 256) +
           round_up(mxfp4_block128_scales_bytes(q.N, q.K, q.b_shape), 256) +
           mxfp4_gemm_block128_workspace_bytes(q.M, q.N, q.K);
}

int mxfp4_linear_pass_block128(int pass, const void* a, const void* b, void* out, int64_t T, int64_t in_features,
                               int64_t out_features, int out_dtype, void* workspace, size_t workspace_bytes,
                               void* stream)
{
    if (pass < 0 || pass > 2) return MXFP4_ERR_ENUM;
    if (!a || !b || !out) return MXFP4_ERR_NULL;
    if (out_dtype != MXFP4_OUT_BF16 && out_dtype != MXFP4_OUT_FP32) return MXFP4_ERR_ENUM;
    if (T <= 0 || in_features <= 0 || out_features <= 0 || in_features % 8 != 0 || out_features % 8 != 0)
        return MXFP4_ERR_SHAPE;
    const Pass128 q = pass128(pass, T, in_features, out_features);
    int rc = gemm128_shape_ok(q.M, q.N, q.K);
    if (rc != MXFP4_OK) return rc;
    const int64_t a_tiles = quantize128_tiles(q.ar, q.ac), b_tiles = quantize128_tiles(q.br, q.bc);
    if (a_tiles > 0x3FFFFFFF || b_tiles > 0x3FFFFFFF) return MXFP4_ERR_SHAPE;
    const size_t need = mxfp4_linear_pass_block128_workspace_bytes(T, in_features, out_features, pass);
    if (!workspace || workspace_bytes < need) return MXFP4_ERR_WORKSPACE;
    if ((reinterpret_cast<uintptr_t>(workspace) & 255u) || !aligned16(a) || !aligned16(b) || !aligned16(out))
        return MXFP4_ERR_ALIGN;
    const DeviceInfo& dev = device_info();
    if ((rc = device_status_code(dev)) != MXFP4_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    uint8_t* a_codes = static_cast<uint8_t*>(workspace);
    uint8_t* a_scales = a_codes + round_up(static_cast<size_t>(q.M) * q.K, 256);
    uint8_t* b_codes = a_scales + round_up(mxfp4_block128_scales_bytes(q.M, q.K, MXFP4_BLOCK_1X128), 256);
    uint8_t* b_scales = b_codes + round_up(static_cast<size_t>(q.N) * q.K, 256);
    uint8_t* parts = b_scales + round_up(mxfp4_block128_scales_bytes(q.N, q.K, q.b_shape), 256);
    // every reduction size is a multiple of 16 by now: one launch quantizes both operands
    const bool square = q.b_shape == MXFP4_BLOCK_128X128;
    const Quant128Params pa = quantize128_params(a, q.ar, q.ac, q.ac, q.a_axis, false, a_codes, a_scales);
    const Quant128Params pb = quantize128_params(b, q.br, q.bc, q.bc, q.b_axis, square, b_codes, b_scales);
    auto kernel = pass == MXFP4_PASS_FPROP ? quantize_block128_both_kernel<1, 1, true>
                  : pass == MXFP4_PASS_DGRAD ? quantize_block128_both_kernel<1, 0, true>
                                             : quantize_block128_both_kernel<0, 0, false>;
    if (launch_kernel_pdl(kernel, static_cast<int>(a_tiles + b_tiles), kB128Threads, 0, st, pa, pb,
                          static_cast<int>(a_tiles)) != cudaSuccess)
        return MXFP4_ERR_CUDA;
    return gemm128_launch(a_codes, a_scales, b_codes, b_scales, q.b_shape == MXFP4_BLOCK_1X128, q.M, q.N, q.K, out,
                          out_dtype, q.N, parts, dev.sm_count, st);
}

}  // extern "C"
