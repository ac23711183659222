// 8-bit quantizer with one fp32 scale per 128 elements along the reduction axis (1 x 128 blocks) or per
// 128 x 128 block, for either axis of the source:
//     a = max(amax, 2^-100),  scale = a / 448,  code = E4M3(x * (448 / a)),  fp32 steps rounded to nearest.
//
// A CTA takes one 128 x 128 tile of the source, each thread eight 16-byte pieces of it, so a tile is
// 32 KB of loads in flight at once and the block maximum never leaves the CTA.  Row-wise blocks
// reduce over the 16 lanes that hold a row.  For the transposed operand a thread holds eight
// consecutive rows of eight columns: eight codes of a column are one 8-byte word of the operand row,
// staged in shared memory (word index XOR-ed with the column group: no bank conflicts either way)
// and written as 16-byte pieces of 128-byte operand rows.
//
// Bound by memory, 3 bytes per element: 8192 x 14336 in 57 (square), 59 (row-wise) and 64 us (transposed) by itself, 5.5
// to 6.1 TB/s; 8192 x 4096 in 23 to 25 us.  What was in the way was the number of instructions per element:
// maxima in fp32, a division per row in each of its sixteen lanes and three CTAs per SM took 64, 79 and 70 us.
// Now maxima are pairs of 16-bit words, two rows share a shuffle, and each lane divides for one row.
#pragma once

#include <cuda_bf16.h>

#include "../../include/mxfp4.h"
#include "ptx_sm100.cuh"
#include "row_io.cuh"

namespace mxfp4 {

constexpr int kB128 = 128;
constexpr int kB128Threads = 256;
constexpr int kB128Ctas = 4;                 // per SM
constexpr float kE4m3Max = 448.0f;
constexpr float kBlockTiny = 7.888609052210118e-31f;      // 2^-100

struct Quant128Params {
    const __nv_bfloat16* src;
    uint8_t* codes;
    float* scales;
    int64_t ld;
    int32_t rows, cols;          // of the source
    int32_t tiles_c;             // tiles along the columns
    int32_t pitch;               // scales of one block along K: 128 * ceil(outer / 128), or ceil(outer / 128)
};

// Eight bf16 of a source row at column `col`; zeros past the edges.
__device__ __forceinline__ uint4 load_piece(const Quant128Params& p, int row, int col)
{
    uint4 w = make_uint4(0u, 0u, 0u, 0u);
    if (row >= p.rows || col >= p.cols) return w;
    const __nv_bfloat16* at = p.src + static_cast<int64_t>(row) * p.ld + col;
    if (col + 8 <= p.cols) return ld_stream(at);
    uint32_t v[4] = {0u, 0u, 0u, 0u};                     // a ragged last piece, element by element
    const uint16_t* e = reinterpret_cast<const uint16_t*>(at);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (col + i < p.cols) v[i >> 1] |= static_cast<uint32_t>(e[i]) << (16 * (i & 1));
    return make_uint4(v[0], v[1], v[2], v[3]);
}

__device__ __forceinline__ uint32_t word_of(const uint4& w, int i)
{
    return i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w;
}

// Magnitudes of bf16 numbers order as their bits do: maxima are taken on pairs of 16-bit words.  A NaN's are above all
// others, and max_nan keeps it: one NaN makes its block's scale and codes NaN.
__device__ __forceinline__ uint32_t magnitudes(uint32_t pair) { return pair & 0x7FFF7FFFu; }
__device__ __forceinline__ uint32_t fold(uint32_t m) { return __vmaxu2(m, m >> 16) & 0xFFFFu; }
__device__ __forceinline__ float magnitude(uint32_t m) { return __uint_as_float(m << 16); }

// largest magnitudes of a piece's even and odd elements
__device__ __forceinline__ uint32_t piece_amax(const uint4& w)
{
    return __vmaxu2(__vmaxu2(magnitudes(w.x), magnitudes(w.y)), __vmaxu2(magnitudes(w.z), magnitudes(w.w)));
}

__device__ __forceinline__ float block_inverse(float amax) { return __fdiv_rn(kE4m3Max, max_nan(amax, kBlockTiny)); }
__device__ __forceinline__ float block_scale(float amax) { return __fdiv_rn(max_nan(amax, kBlockTiny), kE4m3Max); }

__device__ __forceinline__ uint2 piece_codes(const uint4& w, float inv)
{
    return make_uint2(cvt_e4m3x4(bf16_lo(w.x) * inv, bf16_hi(w.x) * inv, bf16_lo(w.y) * inv, bf16_hi(w.y) * inv),
                      cvt_e4m3x4(bf16_lo(w.z) * inv, bf16_hi(w.z) * inv, bf16_lo(w.w) * inv, bf16_hi(w.w) * inv));
}

// AXIS 1: operand row = source row; AXIS 0: operand row = source column.  SQUARE: 128 x 128 blocks.
template <int AXIS, bool SQUARE>
__device__ __forceinline__ void quantize_block128_tile(const Quant128Params& p, int tile)
{
    __shared__ __align__(16) uint8_t codes_t[AXIS == 0 ? kB128 * kB128 : 16];      // [source column][source row]
    __shared__ __align__(16) uint32_t part[AXIS == 0 && !SQUARE ? 16 * kB128 / 2 : 16];    // maxima
    __shared__ __align__(16) float inverse[AXIS == 0 && !SQUARE ? kB128 : 4];              // 448 / maximum, per column
    const int tid = threadIdx.x;
    const int cg = tid & 15, rg = tid >> 4;              // column group of 8, row group
    const int tr = tile / p.tiles_c, tc = tile % p.tiles_c;
    const int row0 = tr * kB128, col0 = tc * kB128;
    // row-wise: rows rg, rg + 16, ...; transposed: rows 8 * rg ... 8 * rg + 7
    auto row_of = [&](int i) { return AXIS == 1 ? rg + 16 * i : 8 * rg + i; };
    uint4 w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = load_piece(p, row0 + row_of(i), col0 + 8 * cg);

    if (SQUARE) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = __vmaxu2(m, piece_amax(w[i]));
        m = __reduce_max_sync(0xffffffffu, fold(m));
        if ((tid & 31) == 0) smem_put(part, tid >> 5, m);
        __syncthreads();
        m = smem_get(part, 0);
#pragma unroll
        for (int i = 1; i < kB128Threads / 32; ++i) m = max(m, smem_get(part, i));
        const float amax = magnitude(m), inv = block_inverse(amax);
        if (tid == 0) {
            const int ob = AXIS == 1 ? tr : tc, kb = AXIS == 1 ? tc : tr;
            p.scales[static_cast<int64_t>(kb) * p.pitch + ob] = block_scale(amax);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint2 c = piece_codes(w[i], inv);
            w[i].x = c.x;
            w[i].y = c.y;
        }
    } else if (AXIS == 1) {
        // two rows' maxima travel in one word; lane cg of a row's sixteen keeps the one of row cg (mod 8) and divides for it
        uint32_t mine = 0;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            uint32_t m = fold(piece_amax(w[i])) | (fold(piece_amax(w[i + 1])) << 16);
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, o));
            if ((cg & 6) == i) mine = (cg & 1) ? m >> 16 : m & 0xFFFFu;
        }
        const float amax = magnitude(mine), inv = block_inverse(amax);
        if (cg < 8) {
            const int row = row0 + row_of(cg);
            p.scales[static_cast<int64_t>(tc) * p.pitch + row] = row < p.rows ? block_scale(amax) : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint2 c = piece_codes(w[i], __shfl_sync(0xffffffffu, inv, i, 16));
            w[i].x = c.x;
            w[i].y = c.y;
        }
    } else {
        // maximum of each column: this thread's eight rows, then the sixteen row groups
        uint32_t m[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            m[j] = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m[j] = __vmaxu2(m[j], magnitudes(word_of(w[i], j)));
        }
        smem_store(part + rg * (kB128 / 2) + cg * 4, make_uint4(m[0], m[1], m[2], m[3]), part, sizeof(part));
        __syncthreads();
        if (tid < kB128) {
            uint32_t a = 0;
#pragma unroll
            for (int g = 0; g < 16; ++g) a = __vmaxu2(a, smem_get(part, g * (kB128 / 2) + (tid >> 1)));
            const float amax = magnitude((tid & 1) ? a >> 16 : a & 0xFFFFu);
            const int col = col0 + tid;
            p.scales[static_cast<int64_t>(tr) * p.pitch + col] = col < p.cols ? block_scale(amax) : 0.0f;
            smem_put(inverse, tid, block_inverse(amax));
        }
        __syncthreads();
        const float4 lo = smem_load<float4>(inverse + cg * 8, inverse, sizeof(inverse));
        const float4 hi = smem_load<float4>(inverse + cg * 8 + 4, inverse, sizeof(inverse));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint4 v = w[i];
            w[i].x = cvt_e4m3x4(bf16_lo(v.x) * lo.x, bf16_hi(v.x) * lo.y, bf16_lo(v.y) * lo.z, bf16_hi(v.y) * lo.w);
            w[i].y = cvt_e4m3x4(bf16_lo(v.z) * hi.x, bf16_hi(v.z) * hi.y, bf16_lo(v.w) * hi.z, bf16_hi(v.w) * hi.w);
        }
    }

    if (AXIS == 1) {
        // codes of a row piece: 8 bytes, 128 contiguous bytes per 16 lanes (cols is a multiple of 16)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = row0 + row_of(i), col = col0 + 8 * cg;
            if (row < p.rows && col < p.cols)
                *reinterpret_cast<uint2*>(p.codes + static_cast<int64_t>(row) * p.cols + col) = make_uint2(w[i].x, w[i].y);
        }
    } else {
        // eight codes of one column -> one 8-byte word: a byte transpose of 8 x 8 in registers
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t r[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) r[i] = half ? w[i].y : w[i].x;
            // columns 0, 1 / 2, 3 of two rows side by side, then four rows of one column
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const uint32_t a = prmt(r[4 * q], r[4 * q + 1], 0x5140u), b = prmt(r[4 * q + 2], r[4 * q + 3], 0x5140u);
                const uint32_t c = prmt(r[4 * q], r[4 * q + 1], 0x7362u), d = prmt(r[4 * q + 2], r[4 * q + 3], 0x7362u);
                r[4 * q] = prmt(a, b, 0x5410u);
                r[4 * q + 1] = prmt(a, b, 0x7632u);
                r[4 * q + 2] = prmt(c, d, 0x5410u);
                r[4 * q + 3] = prmt(c, d, 0x7632u);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int col = cg * 8 + half * 4 + j;
                smem_store(codes_t + col * kB128 + ((rg ^ cg) * 8), make_uint2(r[j], r[4 + j]), codes_t, kB128 * kB128);
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int piece = tid + i * kB128Threads;    // 128 columns x 8 pieces of 16 bytes
            const int col = piece >> 3, c = piece & 7, sw = col >> 3;
            const uint2 lo = smem_load<uint2>(codes_t + col * kB128 + (((2 * c) ^ sw) * 8), codes_t, kB128 * kB128);
            const uint2 hi = smem_load<uint2>(codes_t + col * kB128 + (((2 * c + 1) ^ sw) * 8), codes_t, kB128 * kB128);
            const int o = col0 + col, k = row0 + 16 * c;  // rows is a multiple of 16
            if (o < p.cols && k < p.rows)
                *reinterpret_cast<uint4*>(p.codes + static_cast<int64_t>(o) * p.rows + k) = make_uint4(lo.x, lo.y, hi.x, hi.y);
        }
    }
}

template <int AXIS, bool SQUARE>
__global__ void __launch_bounds__(kB128Threads, kB128Ctas)
quantize_block128_kernel(const Quant128Params p)
{
    griddep_launch_dependents();
    griddep_wait();
    quantize_block128_tile<AXIS, SQUARE>(p, blockIdx.x);
}

// Both operands of a linear's pass in one launch: 1 x 128 blocks of a, then b.
template <int AXIS_A, int AXIS_B, bool SQUARE_B>
__global__ void __launch_bounds__(kB128Threads, kB128Ctas)
quantize_block128_both_kernel(const __grid_constant__ Quant128Params a, const __grid_constant__ Quant128Params b, int a_tiles)
{
    griddep_launch_dependents();
    griddep_wait();
    const int tile = blockIdx.x;
    if (tile < a_tiles) quantize_block128_tile<AXIS_A, false>(a, tile);
    else quantize_block128_tile<AXIS_B, SQUARE_B>(b, tile - a_tiles);
}

}  // namespace mxfp4
