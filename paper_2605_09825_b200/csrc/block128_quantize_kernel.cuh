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
#pragma once

#include <cuda_bf16.h>

#include "../../include/mxfp4.h"
#include "ptx_sm100.cuh"
#include "row_io.cuh"

namespace mxfp4 {

constexpr int kB128 = 128;
constexpr int kB128Threads = 256;
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

// largest magnitude of the eight values, as fp32
__device__ __forceinline__ float piece_amax(const uint4& w)
{
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = fmaxf(m, fmaxf(fabsf(bf16_lo(word_of(w, i))), fabsf(bf16_hi(word_of(w, i)))));
    return m;
}

__device__ __forceinline__ float block_inverse(float amax) { return __fdiv_rn(kE4m3Max, fmaxf(amax, kBlockTiny)); }
__device__ __forceinline__ float block_scale(float amax) { return __fdiv_rn(fmaxf(amax, kBlockTiny), kE4m3Max); }

__device__ __forceinline__ uint2 piece_codes(const uint4& w, float inv)
{
    return make_uint2(cvt_e4m3x4(bf16_lo(w.x) * inv, bf16_hi(w.x) * inv, bf16_lo(w.y) * inv, bf16_hi(w.y) * inv),
                      cvt_e4m3x4(bf16_lo(w.z) * inv, bf16_hi(w.z) * inv, bf16_lo(w.w) * inv, bf16_hi(w.w) * inv));
}

// AXIS 1: operand row = source row; AXIS 0: operand row = source column.  SQUARE: 128 x 128 blocks.
template <int AXIS, bool SQUARE>
__global__ void __launch_bounds__(kB128Threads, 3) quantize_block128_kernel(const Quant128Params p)
{
    __shared__ __align__(16) uint8_t codes_t[AXIS == 0 ? kB128 * kB128 : 16];      // [source column][source row]
    __shared__ float part[AXIS == 0 && !SQUARE ? 16 * kB128 : 16];
    griddep_launch_dependents();
    griddep_wait();
    const int tid = threadIdx.x;
    const int cg = tid & 15, rg = tid >> 4;              // column group of 8, row group
    const int tr = blockIdx.x / p.tiles_c, tc = blockIdx.x % p.tiles_c;
    const int row0 = tr * kB128, col0 = tc * kB128;
    // row-wise: rows rg, rg + 16, ...; transposed: rows 8 * rg ... 8 * rg + 7
    auto row_of = [&](int i) { return AXIS == 1 ? rg + 16 * i : 8 * rg + i; };
    uint4 w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = load_piece(p, row0 + row_of(i), col0 + 8 * cg);

    if (SQUARE) {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaxf(m, piece_amax(w[i]));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        if ((tid & 31) == 0) part[tid >> 5] = m;
        __syncthreads();
        m = part[0];
#pragma unroll
        for (int i = 1; i < kB128Threads / 32; ++i) m = fmaxf(m, part[i]);
        const float inv = block_inverse(m);
        if (tid == 0) {
            const int ob = AXIS == 1 ? tr : tc, kb = AXIS == 1 ? tc : tr;
            p.scales[static_cast<int64_t>(kb) * p.pitch + ob] = block_scale(m);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint2 c = piece_codes(w[i], inv);
            w[i].x = c.x;
            w[i].y = c.y;
        }
    } else if (AXIS == 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float m = piece_amax(w[i]);
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            const int row = row0 + row_of(i);
            if (cg == 0) p.scales[static_cast<int64_t>(tc) * p.pitch + row] = row < p.rows ? block_scale(m) : 0.0f;
            const uint2 c = piece_codes(w[i], block_inverse(m));
            w[i].x = c.x;
            w[i].y = c.y;
        }
    } else {
        // maximum of each column: this thread's eight rows, then the sixteen row groups
        float m[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            m[j] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t v = word_of(w[i], j >> 1);
                m[j] = fmaxf(m[j], fabsf((j & 1) ? bf16_hi(v) : bf16_lo(v)));
            }
        }
#pragma unroll
        for (int j = 0; j < 8; j += 4)
            *reinterpret_cast<float4*>(&part[rg * kB128 + cg * 8 + j]) = make_float4(m[j], m[j + 1], m[j + 2], m[j + 3]);
        __syncthreads();
        if (tid < kB128) {
            float a = 0.0f;
#pragma unroll
            for (int g = 0; g < 16; ++g) a = fmaxf(a, part[g * kB128 + tid]);
            const int col = col0 + tid;
            p.scales[static_cast<int64_t>(tr) * p.pitch + col] = col < p.cols ? block_scale(a) : 0.0f;
            part[tid] = block_inverse(a);                 // row group 0's maxima of this column: read above, by this thread
        }
        __syncthreads();
        float inv[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) inv[j] = part[cg * 8 + j];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint4 v = w[i];
            w[i].x = cvt_e4m3x4(bf16_lo(v.x) * inv[0], bf16_hi(v.x) * inv[1], bf16_lo(v.y) * inv[2], bf16_hi(v.y) * inv[3]);
            w[i].y = cvt_e4m3x4(bf16_lo(v.z) * inv[4], bf16_hi(v.z) * inv[5], bf16_lo(v.w) * inv[6], bf16_hi(v.w) * inv[7]);
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

}  // namespace mxfp4
