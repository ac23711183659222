// The 128-block product for few rows of A (decoding steps): out[m][n] for m < 8 * TILES, bound by reading B once.
//
// A CTA takes 16 rows of B, its eight warps take K-blocks of 128 in turn and add their sums through shared
// memory in a fixed order.  The products run on mma.sync m16n8k32 with B's rows as the instruction's 16 rows
// and A's as its eight columns: what the instruction cannot reach in rate does not matter here, and it needs
// neither staging nor tensor memory.  The order of the 32 elements inside an instruction is free as long as
// both operands agree, so a lane's 16-byte pieces of a row go in as they come: a quad covers 64 contiguous
// bytes of each row.  Every K-block is a product of its own, scaled and added in fp32.
//
// Codes and scales of two K-blocks are loaded before the first product: two CTAs of eight warps keep 64 KB of B in
// flight per SM.  1 x 4096 x 14336: 13.4 us (58.7 MB, 4.4 TB/s, with two launches' worth of latency in it),
// 1 x 128256 x 4096: 92 us (5.7 TB/s); 16 rows: 16.8 and 120 us, the rows of A coming from L2 once per CTA.
// Scales loaded where they are used: 14.0 and 98.6 us; four K-blocks in flight: 13.8 and 86 us, but 15.2
// and 103 with a scale per row of B and 138 with 16 rows (registers); three or four CTAs per SM spill; 32 rows of B
// per CTA: 20 and 88 us; a persistent grid with a ring of asynchronous copies in shared memory: 17 to 25 and
// 101 to 127 us.
#pragma once

#include <cuda_bf16.h>

#include "../../include/mxfp4.h"
#include "ptx_sm100.cuh"

namespace mxfp4 {

constexpr int kRowsWarps = 8;
constexpr int kRowsB = 16;                       // rows of B per CTA
constexpr int kRowsMaxTiles = 2;                 // of eight rows of A each

struct Rows128Params {
    const uint8_t* a_codes;
    const uint8_t* b_codes;
    const float* a_scales;
    const float* b_scales;
    void* out;
    int64_t ld_out;
    int64_t pitch_a, pitch_b;
    int32_t M, N, K;
    int32_t k_blocks;
    int32_t out_fp32;
};

__device__ __forceinline__ uint4 ldg16(const uint8_t* p, bool valid)
{
    return valid ? __ldg(reinterpret_cast<const uint4*>(p)) : make_uint4(0u, 0u, 0u, 0u);
}

// read once: past L1
__device__ __forceinline__ uint4 ldg16_stream(const uint8_t* p, bool valid)
{
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (valid)
        asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                     : "l"(p));
    return v;
}

__device__ __forceinline__ void mma_e4m3_16x8x32(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                 uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <bool BROWS, int TILES>
__global__ void __launch_bounds__(kRowsWarps * 32, 2) gemm_block128_rows_kernel(const __grid_constant__ Rows128Params p)
{
    __shared__ float part[kRowsWarps][TILES][4][32];
    griddep_launch_dependents();
    griddep_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, q = lane & 3;           // row of the fragment (and of A), quarter of a 64-byte piece
    const int n0 = blockIdx.x * kRowsB;
    const bool row0 = n0 + g < p.N, row1 = n0 + g + 8 < p.N;
    const uint8_t* b0 = p.b_codes + static_cast<int64_t>(n0 + g) * p.K;
    const uint8_t* b1 = b0 + static_cast<int64_t>(8) * p.K;
    float acc[TILES][4];
#pragma unroll
    for (int m = 0; m < TILES; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[m][i] = 0.0f;

    // K-blocks in flight per warp.  A step's second block may start past K; its number is 8 to 15 modulo 16 and its first
    // block's at most 2^24 - 3, so it is below 2^24, and element numbers stay below 2^31
    constexpr int kUnroll = 2;
    for (int t0 = warp; t0 < p.k_blocks; t0 += kUnroll * kRowsWarps) {
        uint4 w0[kUnroll][2], w1[kUnroll][2], x[kUnroll][TILES][2];
        float2 sa[kUnroll][TILES];
        float sb0[kUnroll], sb1[kUnroll];
        // everything the blocks need is on its way before the first product
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int t = t0 + u * kRowsWarps;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = t * 128 + h * 64 + q * 16;
                w0[u][h] = ldg16_stream(b0 + k, row0 && k < p.K);
                w1[u][h] = ldg16_stream(b1 + k, row1 && k < p.K);
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int t = t0 + u * kRowsWarps;
            const bool in = t < p.k_blocks;
#pragma unroll
            for (int m = 0; m < TILES; ++m) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int k = t * 128 + h * 64 + q * 16, row = m * 8 + g;
                    x[u][m][h] = ldg16(p.a_codes + static_cast<int64_t>(row) * p.K + k, row < p.M && k < p.K);
                }
                // the scales of A reach to 128 rows
                sa[u][m] = in ? __ldg(reinterpret_cast<const float2*>(p.a_scales + t * p.pitch_a + m * 8 + 2 * q))
                              : make_float2(0.0f, 0.0f);
            }
            if (BROWS) {
                sb0[u] = row0 && in ? __ldg(p.b_scales + t * p.pitch_b + n0 + g) : 0.0f;
                sb1[u] = row1 && in ? __ldg(p.b_scales + t * p.pitch_b + n0 + g + 8) : 0.0f;
            } else {
                sb0[u] = sb1[u] = in ? __ldg(p.b_scales + t * p.pitch_b + n0 / 128) : 0.0f;
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int m = 0; m < TILES; ++m) {
                float c[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint4 v = x[u][m][h];
                    mma_e4m3_16x8x32(c, w0[u][h].x, w1[u][h].x, w0[u][h].y, w1[u][h].y, v.x, v.y);
                    mma_e4m3_16x8x32(c, w0[u][h].z, w1[u][h].z, w0[u][h].w, w1[u][h].w, v.z, v.w);
                }
                // this lane's sums: rows g and g + 8 of B, rows 2 q and 2 q + 1 of A
                acc[m][0] = fmaf(c[0], sa[u][m].x * sb0[u], acc[m][0]);
                acc[m][1] = fmaf(c[1], sa[u][m].y * sb0[u], acc[m][1]);
                acc[m][2] = fmaf(c[2], sa[u][m].x * sb1[u], acc[m][2]);
                acc[m][3] = fmaf(c[3], sa[u][m].y * sb1[u], acc[m][3]);
            }
    }
#pragma unroll
    for (int m = 0; m < TILES; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) smem_store(&part[warp][m][i][lane], acc[m][i], part, sizeof(part));
    __syncthreads();
    for (int e = threadIdx.x; e < TILES * 128; e += kRowsWarps * 32) {
        const int m = e >> 7, i = (e >> 5) & 3, l = e & 31;
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kRowsWarps; ++w) s += smem_load<float>(&part[w][m][i][l], part, sizeof(part));
        const int row = m * 8 + 2 * (l & 3) + (i & 1), col = n0 + (l >> 2) + 8 * (i >> 1);
        if (row < p.M && col < p.N) {
            const int64_t at = row * p.ld_out + col;
            if (p.out_fp32) static_cast<float*>(p.out)[at] = s;
            else static_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(s);
        }
    }
}

}  // namespace mxfp4
