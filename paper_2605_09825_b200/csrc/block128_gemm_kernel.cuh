// 8-bit product with one fp32 scale per 128 elements along K:
//
//   out[m][n] = sum_t sa[t][m] * sb[t][n or n / 128] * sum_{k in block t} A[m][k] * B[n][k]
//
// CTA-pair kernel (tcgen05 cta_group::2) on 256 x 256 output tiles.  The scales are not powers of two, so the
// tensor cores cannot apply them: each K-step of 128 elements is a product of its own, formed in one
// of two TMEM buffers (2 x 256 columns: all of TMEM) while the epilogue warps read the other one and add
// it, scaled, to sums they keep in registers -- 128 rows x 256 columns per CTA, 128 sums per thread.
// Four K = 32 instructions are the longest chain of the tensor cores' truncating additions.
//
// Per SM and K-step: 512 cycles of MMA; 128 x 256 multiply-adds of the epilogue, packed in pairs, are 256
// cycles of the FMA pipe (twice that when B has a scale per row, which costs a multiplication per
// element more) and 256 cycles of tensor-memory reads beside it.
//
// Roles per CTA (384 threads): warps 0..7 epilogue (32 rows x 128 columns each), warp 8 TMA producer,
// warp 9 MMA issuer (leader CTA only).  Barrier ownership as in the block-scaled kernel: full and
// tmem_empty live in the leader, empty and tmem_full are signalled in both CTAs by a multicast
// commit.  All waits are bounded.
//
// Products with few output tiles are split along K (`splits`): each split writes its fp32 sums to
// the workspace and a second kernel adds them in a fixed order.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>

#include "../../include/mxfp4.h"
#include "ptx_sm100.cuh"
#include "tma_host.cuh"

namespace mxfp4 {

constexpr int kBTile = 256;                       // both ways
constexpr int kBHalf = 128;                       // rows of A, and of B, per CTA
constexpr int kBBlockK = 128;                     // elements = bytes per stage and row
constexpr int kBStages = 5;
constexpr int kBOperandBytes = kBHalf * kBBlockK; // 16 KB
constexpr int kBEpiWarps = 8;
constexpr int kBProducerWarp = 8;
constexpr int kBMmaWarp = 9;
constexpr int kBThreads = 384;
constexpr int kBStageBytes = 32 * 128;            // output staging per epilogue warp

struct Gemm128Smem {
    alignas(1024) uint8_t a[kBStages][kBOperandBytes];
    alignas(1024) uint8_t b[kBStages][kBOperandBytes];
    alignas(1024) uint8_t out_stage[kBEpiWarps][kBStageBytes];
    alignas(16) float sb[kBEpiWarps][2][kBHalf];  // this K-step's scales of the warp's 128 columns
    alignas(8) uint64_t full[kBStages];           // leader's copy is the live one
    uint64_t empty[kBStages];                     // both, via multicast commit
    uint64_t tmem_full[2];                        // both, via multicast commit
    uint64_t tmem_empty[2];                       // leader's copy is the live one
    uint32_t tmem_base;
    int abort_flag;
};

struct Gemm128Params {
    const float* a_scales;
    const float* b_scales;
    void* out;                   // for the columns past the last 16-byte granule
    int64_t ld_out;
    int64_t split_stride;        // elements between the splits' outputs
    int64_t pitch_a;             // scales per K-step of A, of B
    int64_t pitch_b;
    int32_t M, N, K;
    int32_t tiles_m, tiles_n;
    int32_t band;                // tile columns per band of the tile order
    int32_t k_steps;             // ceil(K / 128)
    int32_t splits;              // along K
    int32_t n_tma;               // columns written by TMA stores
};

// A piece of work: one output tile, one range of K-steps.  Tiles are numbered band by band: a band is
// `band` tile columns, sized so that its B panel stays in L2, and inside a band the tile column varies
// fastest, so that the tiles in flight share A rows and B columns.
struct Gemm128Work {
    int tm, tn, split, k0, k1;
};

__device__ __forceinline__ Gemm128Work gemm128_work(const Gemm128Params& p, int item)
{
    Gemm128Work w;
    const int tile = item / p.splits;
    w.split = item - tile * p.splits;
    const int per_band = p.band * p.tiles_m;
    const int b = tile / per_band;
    const int r = tile - b * per_band;
    const int cols = min(p.band, p.tiles_n - b * p.band);
    w.tm = r / cols;
    w.tn = b * p.band + (r - w.tm * cols);
    w.k0 = static_cast<int>(static_cast<int64_t>(p.k_steps) * w.split / p.splits);
    w.k1 = static_cast<int>(static_cast<int64_t>(p.k_steps) * (w.split + 1) / p.splits);
    return w;
}

// Columns the MMAs of a tile column compute: what exists, rounded up to the instruction's granule.
__device__ __forceinline__ int gemm128_width(int N, int tn) { return min(kBTile, (N - tn * kBTile + 15) & ~15); }

// BROWS: B has a scale per row and K-step (1 x 128 blocks); otherwise one per 128 rows.
template <bool BROWS, bool OUT32>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kBThreads, 1)
gemm_block128_pair_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b,
                          const __grid_constant__ CUtensorMap tm_out, const Gemm128Params p)
{
    extern __shared__ uint8_t smem_raw[];
    Gemm128Smem& sm = *reinterpret_cast<Gemm128Smem*>(smem_align_1024(smem_raw));
    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int cluster_id = blockIdx.x >> 1;
    const int n_clusters = gridDim.x >> 1;
    const int items = p.tiles_m * p.tiles_n * p.splits;

    if (threadIdx.x == 0) {
        sm.abort_flag = 0;
        for (int s = 0; s < kBStages; ++s) {
            mbar_init(&sm.full[s], 2);                 // one arrive.expect_tx per CTA
            mbar_init(&sm.empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&sm.tmem_full[b], 1);
            mbar_init(&sm.tmem_empty[b], 2 * kBEpiWarps);
        }
        fence_barrier_init();
    }
    if (warp == kBMmaWarp) {
        tmem_alloc_pair(&sm.tmem_base, 512);
        tmem_relinquish_pair();
    }
    tcgen05_fence_before();
    __syncthreads();
    cluster_sync_all();           // both CTAs' barriers exist before anyone signals across the pair
    tcgen05_fence_after();
    const uint32_t tmem = sm.tmem_base;
    griddep_launch_dependents();
    griddep_wait();

    // registers: 384 x 168 at launch = 256 x 208 (epilogue) + 128 x 88 (the others)
    if (warp >= kBEpiWarps) {
        setmaxnreg_dec<88>();
        if (warp == kBProducerWarp) {
            // -------------------------------------------------------- TMA producer
            if (lane == 0) {
                tma_prefetch_desc(&tm_a);
                tma_prefetch_desc(&tm_b);
            }
            int it = 0;
            bool alive = true;
            for (int item = cluster_id; alive && item < items; item += n_clusters) {
                const Gemm128Work w = gemm128_work(p, item);
                const int32_t ya = w.tm * kBTile + static_cast<int>(rank) * kBHalf;
                // this CTA's share of the MMA's rows of B; the box is always 128 rows
                const int32_t yb = w.tn * kBTile + static_cast<int>(rank) * (gemm128_width(p.N, w.tn) >> 1);
                for (int k = w.k0; k < w.k1; ++k, ++it) {
                    const int s = it % kBStages;
                    const uint32_t round = it / kBStages;
                    if (round > 0 && !mbar_wait(&sm.empty[s], (round - 1) & 1, &sm.abort_flag)) {
                        alive = false;
                        break;
                    }
                    if (elect_one_sync()) {
                        const uint32_t full_leader = map_to_cta(smem_u32(&sm.full[s]), 0);
                        mbar_arrive_expect_tx_cluster(full_leader, 2 * kBOperandBytes);
                        tma_load_2d_pair(sm.a[s], &tm_a, full_leader, k * kBBlockK, ya);
                        tma_load_2d_pair(sm.b[s], &tm_b, full_leader, k * kBBlockK, yb);
                    }
                    __syncwarp();
                }
            }
        } else if (warp == kBMmaWarp && rank == 0) {
            // -------------------------------------------------------- MMA issuer
            const uint64_t a_desc0 = make_smem_desc(smem_u32(sm.a[0]), 16, 1024, 2);
            const uint64_t b_desc0 = make_smem_desc(smem_u32(sm.b[0]), 16, 1024, 2);
            int it = 0;
            bool alive = true;
            for (int item = cluster_id; alive && item < items; item += n_clusters) {
                const Gemm128Work w = gemm128_work(p, item);
                // instruction descriptor: fp32 accumulator, E4M3 x E4M3, K-major operands
                const uint32_t idesc = (1u << 4) | (static_cast<uint32_t>(gemm128_width(p.N, w.tn) >> 3) << 17) |
                                       (static_cast<uint32_t>(kBTile >> 4) << 24);
                for (int k = w.k0; k < w.k1; ++k, ++it) {
                    const int s = it % kBStages, b = it & 1;
                    if (!mbar_wait(&sm.full[s], (it / kBStages) & 1, &sm.abort_flag) ||
                        (it >= 2 && !mbar_wait(&sm.tmem_empty[b], ((it >> 1) - 1) & 1, &sm.abort_flag))) {
                        alive = false;
                        break;
                    }
                    tcgen05_fence_after();
                    const int nmma = (min(kBBlockK, p.K - k * kBBlockK) + 31) / 32;
                    if (elect_one_sync()) {
                        const uint64_t a_desc = a_desc0 + static_cast<uint64_t>(s * (kBOperandBytes >> 4));
                        const uint64_t b_desc = b_desc0 + static_cast<uint64_t>(s * (kBOperandBytes >> 4));
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (j < nmma)
                                tcgen05_mma_f8_pair(tmem + b * kBTile, a_desc + 2 * j, b_desc + 2 * j, idesc, j > 0);
                        tcgen05_commit_pair(&sm.empty[s], 3);
                        tcgen05_commit_pair(&sm.tmem_full[b], 3);
                    }
                    __syncwarp();
                }
            }
        }
    } else {
        // ------------------------------------------------------------ epilogue warps
        setmaxnreg_inc<208>();
        const int quad = warp & 3;                     // TMEM lane quadrant of this warp
        const int half = warp >> 2;                    // which 128 columns
        uint8_t* stg = sm.out_stage[warp];
        const uint32_t taddr0 = tmem + (static_cast<uint32_t>(quad * 32) << 16) + half * kBHalf;
        const uint32_t tmem_empty_leader = map_to_cta(smem_u32(&sm.tmem_empty[0]), 0);
        int it = 0;
        bool alive = true;
        for (int item = cluster_id; alive && item < items; item += n_clusters) {
            const Gemm128Work w = gemm128_work(p, item);
            const int row0 = w.tm * kBTile + static_cast<int>(rank) * kBHalf + quad * 32;
            const int col0 = w.tn * kBTile + half * kBHalf;
            const bool wanted = row0 < p.M && col0 < p.N;        // warp-uniform: something to keep here
            const bool row_ok = row0 + lane < p.M;
            const float* sa_at = p.a_scales + row0 + lane;
            const float* sb_at = p.b_scales + (BROWS ? col0 + lane * 4 : col0 / kBHalf);
            float2 acc[64];
#pragma unroll
            for (int i = 0; i < 64; ++i) acc[i] = make_float2(0.0f, 0.0f);
            // scales one K-step ahead of their use
            float sa_next = 0.0f;
            float4 sb_next = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            auto fetch = [&](int k) {
                if (wanted && k < w.k1) {
                    if (row_ok) sa_next = sa_at[k * p.pitch_a];
                    if (BROWS) sb_next = *reinterpret_cast<const float4*>(sb_at + k * p.pitch_b);
                    else sb_next.x = sb_at[k * p.pitch_b];
                }
            };
            fetch(w.k0);
            for (int k = w.k0; k < w.k1; ++k, ++it) {
                const int b = it & 1;
                const float scale = BROWS ? sa_next : sa_next * sb_next.x;
                float* sb = sm.sb[warp][b];
                if (BROWS) {
                    // the previous reader of this buffer is two steps back, with a warp barrier since
                    smem_store(sb + lane * 4, sb_next, sb, sizeof(sm.sb[warp][b]));
                    __syncwarp();
                }
                fetch(k + 1);
                if (!mbar_wait(&sm.tmem_full[b], (it >> 1) & 1, &sm.abort_flag)) {
                    alive = false;
                    break;
                }
                tcgen05_fence_after();
                if (wanted) {
                    const float2 scale2 = make_float2(scale, scale);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t r[32];
                        tmem_ld_32x32b_x32(taddr0 + b * kBTile + c * 32, r);
                        tmem_ld_wait();
                        if (c == 3) {
                            tcgen05_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive_cluster(tmem_empty_leader + b * 8);
                        }
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            float2 v0 = make_float2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1]));
                            float2 v1 = make_float2(__uint_as_float(r[2 * i + 2]), __uint_as_float(r[2 * i + 3]));
                            if (BROWS) {
                                const float4 q = smem_load<float4>(sb + c * 32 + i * 2, sb, sizeof(sm.sb[warp][b]));
                                v0 = __fmul2_rn(v0, make_float2(q.x, q.y));
                                v1 = __fmul2_rn(v1, make_float2(q.z, q.w));
                            }
                            acc[c * 16 + i] = __ffma2_rn(v0, scale2, acc[c * 16 + i]);
                            acc[c * 16 + i + 1] = __ffma2_rn(v1, scale2, acc[c * 16 + i + 1]);
                        }
                    }
                } else {
                    if (lane == 0) mbar_arrive_cluster(tmem_empty_leader + b * 8);
                }
            }
            if (!alive || !wanted) continue;
            // the warp's 32 rows x 128 columns leave in boxes of 128 bytes per row, staged in the 128-byte
            // swizzle for a TMA store that clips at the matrix edges
            constexpr int kBoxCols = OUT32 ? 32 : 64;
            constexpr int kGranule = OUT32 ? 4 : 8;
#pragma unroll
            for (int c = 0; c < kBHalf / kBoxCols; ++c) {
                const int col = col0 + c * kBoxCols;
                if (lane == 0) bulk_wait_group_read<0>();
                __syncwarp();
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    uint4 v;
                    if (OUT32) {
                        const float2 x = acc[c * 16 + 2 * q], y = acc[c * 16 + 2 * q + 1];
                        v = make_uint4(__float_as_uint(x.x), __float_as_uint(x.y), __float_as_uint(y.x), __float_as_uint(y.y));
                    } else {
                        uint32_t e[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const __nv_bfloat162 h = __floats2bfloat162_rn(acc[c * 32 + 4 * q + j].x, acc[c * 32 + 4 * q + j].y);
                            e[j] = *reinterpret_cast<const uint32_t*>(&h);
                        }
                        v = make_uint4(e[0], e[1], e[2], e[3]);
                    }
                    smem_store(stg + lane * 128 + ((q ^ (lane & 7)) * 16), v, stg, kBStageBytes);
                }
                fence_proxy_async_smem();
                __syncwarp();
                // columns past the last full 16-byte granule, one by one from the staged row
                const int rc = p.n_tma - col;
                if (p.n_tma < p.N && rc >= 0 && rc < kBoxCols && row_ok) {
                    const int q = rc / kGranule;
                    const uint4 v = smem_load<uint4>(stg + lane * 128 + ((q ^ (lane & 7)) * 16), stg, kBStageBytes);
                    const int64_t at = w.split * p.split_stride + static_cast<int64_t>(row0 + lane) * p.ld_out + p.n_tma;
                    const uint32_t e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int j = 0; j < kGranule; ++j)
                        if (p.n_tma + j < p.N) {
                            if (OUT32) static_cast<uint32_t*>(p.out)[at + j] = e[j & 3];
                            else static_cast<uint16_t*>(p.out)[at + j] = static_cast<uint16_t>(e[j >> 1] >> (16 * (j & 1)));
                        }
                }
                if (lane == 0 && col < p.n_tma) {
                    tma_store_3d(&tm_out, stg, col, row0, w.split);
                    bulk_commit_group();
                }
            }
        }
        if (lane == 0) bulk_wait_group<0>();
    }

    // neither CTA may leave (or free TMEM) while its peer can still signal it or read its memory
    tcgen05_fence_before();
    __syncthreads();
    cluster_sync_all();
    if (warp == kBMmaWarp) {
        tcgen05_fence_after();
        tmem_dealloc_pair(tmem, 512);
    }
}

// Sum of the splits' fp32 outputs, in the order of the splits; four columns per thread.
struct Gemm128JoinParams {
    const float* parts;          // [split][M][ld]
    int64_t ld;                  // a multiple of 4
    int64_t split_stride;
    void* out;
    int64_t ld_out;
    int32_t M, N;
    int32_t splits;
    int32_t out_fp32;
};

__global__ void __launch_bounds__(256) gemm_block128_join_kernel(const Gemm128JoinParams p)
{
    griddep_launch_dependents();
    griddep_wait();
    const int64_t quads = p.ld / 4;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t row = at / quads;
    const int col = static_cast<int>(at - row * quads) * 4;
    if (row >= p.M || col >= p.N) return;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int i = 0; i < p.splits; ++i) {
        const float4 v = *reinterpret_cast<const float4*>(p.parts + i * p.split_stride + row * p.ld + col);
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    const float e[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (col + j < p.N) {
            if (p.out_fp32) static_cast<float*>(p.out)[row * p.ld_out + col + j] = e[j];
            else static_cast<__nv_bfloat16*>(p.out)[row * p.ld_out + col + j] = __float2bfloat16_rn(e[j]);
        }
}

}  // namespace mxfp4
