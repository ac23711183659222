// The gated projections for few tokens (decoding steps): h[t][f] for up to eight tokens, bound by reading both weights once.
//
// A CTA takes eight features, its eight warps take pieces of 64 elements of the reduction in turn and add their sums
// through shared memory in a fixed order.  The products run on mma.sync m16n8k16: the instruction's first eight rows are
// the features' rows of the gate's weight, the other eight the same rows of the other weight, its eight columns are
// tokens, so that a thread ends with both projections of the same elements.  What the instruction cannot reach in rate
// does not matter here, and it needs neither staging nor tensor memory.  The order of the 16 elements inside an
// instruction is free as long as both operands agree, so a lane's 16-byte pieces of a row go in as they come: a quad
// covers 64 contiguous bytes of each row.
//
// 4096 x 14336, one token: 36 us for 235 MB, the copy rate; eight tokens 38 us.  Sixteen took 49 us with two tiles of tokens (the
// tokens' rows come from L2 once per CTA, and their registers halve the pieces in flight): the other kernel takes 43.
#pragma once

#include <cuda_bf16.h>

#include "../../include/mxfp4.h"
#include "activations.cuh"
#include "ptx_sm100.cuh"

namespace mxfp4 {

constexpr int kGRowsWarps = 8;
constexpr int kGRowsFeatures = 8;                // per CTA
constexpr int kGRowsTokens = 8;

struct GatedRowsParams {
    const __nv_bfloat16* x;
    const __nv_bfloat16* w_gate;
    const __nv_bfloat16* w_up;
    __nv_bfloat16* h;
    __nv_bfloat16* gate;         // NULL: not kept
    __nv_bfloat16* up;
    int64_t ld_x, ld_gate, ld_up, ld_h, ld_kept;
    int32_t tokens, features, K;
    int32_t act;
};

__device__ __forceinline__ uint4 ldg16_weight(const __nv_bfloat16* p, bool valid)
{
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (valid)
        asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                     : "l"(p));
    return v;
}

__device__ __forceinline__ void mma_bf16_16x8x16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                 uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__global__ void __launch_bounds__(kGRowsWarps * 32, 2) gated_rows_kernel(const __grid_constant__ GatedRowsParams p)
{
    __shared__ float part[kGRowsWarps][4][32];
    griddep_launch_dependents();
    griddep_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, q = lane & 3;           // feature (and token) of the fragment, quarter of a 64-byte piece
    const int f0 = blockIdx.x * kGRowsFeatures;      // features are a multiple of eight: none is missing
    const __nv_bfloat16* wg = p.w_gate + (f0 + g) * p.ld_gate;
    const __nv_bfloat16* wu = p.w_up + (f0 + g) * p.ld_up;
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};

    constexpr int kPiece = 64;                       // elements
    constexpr int kUnroll = 4;                       // pieces in flight per warp
    for (int k0 = warp * kPiece; k0 < p.K; k0 += kUnroll * kGRowsWarps * kPiece) {
        uint4 a[kUnroll][2], b[kUnroll][2], x[kUnroll][2];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = k0 + u * kGRowsWarps * kPiece + h * 32 + q * 8;
                a[u][h] = ldg16_weight(wg + k, k < p.K);
                b[u][h] = ldg16_weight(wu + k, k < p.K);
            }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = k0 + u * kGRowsWarps * kPiece + h * 32 + q * 8;
                x[u][h] = g < p.tokens && k < p.K ? __ldg(reinterpret_cast<const uint4*>(p.x + g * p.ld_x + k))
                                                  : make_uint4(0u, 0u, 0u, 0u);
            }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint4 v = x[u][h];
                mma_bf16_16x8x16(acc, a[u][h].x, b[u][h].x, a[u][h].y, b[u][h].y, v.x, v.y);
                mma_bf16_16x8x16(acc, a[u][h].z, b[u][h].z, a[u][h].w, b[u][h].w, v.z, v.w);
            }
    }
    // this lane's sums: gate (0, 1) and other projection (2, 3) of feature g and tokens 2 q and 2 q + 1
#pragma unroll
    for (int i = 0; i < 4; ++i) smem_store(&part[warp][i][lane], acc[i], part, sizeof(part));
    __syncthreads();
    if (threadIdx.x < 64) {
        // eight threads in turn write a token's eight features
        const int t = threadIdx.x >> 3, f = threadIdx.x & 7;
        const int l = f * 4 + (t >> 1), i = t & 1;
        float gate = 0.0f, up = 0.0f;
#pragma unroll
        for (int w = 0; w < kGRowsWarps; ++w) {
            gate += smem_load<float>(&part[w][i][l], part, sizeof(part));
            up += smem_load<float>(&part[w][i + 2][l], part, sizeof(part));
        }
        const int64_t row = t;
        if (row >= p.tokens) return;
        with_act(p.act, [&](auto act) {
            p.h[row * p.ld_h + f0 + f] = __float2bfloat16_rn(act_value<decltype(act)::value>(gate) * up);
        });
        if (p.gate) {
            p.gate[row * p.ld_kept + f0 + f] = __float2bfloat16_rn(gate);
            p.up[row * p.ld_kept + f0 + f] = __float2bfloat16_rn(up);
        }
    }
}

}  // namespace mxfp4
