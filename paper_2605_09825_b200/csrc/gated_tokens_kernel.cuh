// The gated projections for tens to some hundreds of tokens, and for numbers that fill tiles of 256 badly, with the
// weights as the tensor cores' 256 rows and the tokens as their columns: an instruction for 17 tokens has an eighth of the
// columns of one for 256 (a tile is a multiple of 16 tokens), where the other way round (dense_gemm_kernel.cuh) both cost
// the same, and both weights are read as fast as memory gives them.
//
// CTA-pair kernel (tcgen05 cta_group::2, kind::f16).  A tile is 128 features and up to 256 tokens (a multiple of 16, the same
// for all tiles).  Each CTA holds 64 rows of the gate's weight and the same 64 of the other one -- lanes 0..63 and 64..127
// of its tensor memory -- and half of the tokens, per K-step of 64 elements; as many steps are in flight as fit 160 KB: nine
// for up to 16 tokens, five for 256.  Two accumulators take turns.
//
// Epilogue: chunks of 32 tokens, the even ones for warps 0..3, the odd ones for warps 4..7.  The two warps that hold the other
// projection hand it over through shared memory; the two that hold the gate form h.  Results are staged as rows of 64
// features and leave by TMA stores of 16 tokens, which clip at the last token.
//
// 4096 x 14336, pass after pass, on one device and another: 9 to 64 tokens 41 to 44 us (235 MB, 5.5 TB/s; 112 tiles are one
// round and a half of 74 pairs), 128 tokens 47 to 49, 333 tokens 78 to 91.  With the K-steps of all tiles shared out
// evenly and a joining kernel a call of 17 tokens took 42 + 4.5 us by itself, one of 333 tokens 92 + 20.
//
// Roles per CTA as in the other kernel: warps 0..7 epilogue, 8 TMA producer, 9 MMA issuer (leader CTA only).
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>

#include "../../include/mxfp4.h"
#include "activations.cuh"
#include "ptx_sm100.cuh"
#include "row_io.cuh"

namespace mxfp4 {

constexpr int kTFeatures = 128;                    // per tile and pair
constexpr int kTBlockK = 64;                       // elements: 128 bytes
constexpr int kTWeightBytes = 2 * 64 * 128;        // per CTA and step: 64 rows of both weights
constexpr int kTRing = 160 * 1024;
constexpr int kTMostStages = 9;                     // of 17 KB, the least
constexpr int kTProducerWarp = 8;
constexpr int kTMmaWarp = 9;
constexpr int kTThreads = 320;
constexpr int kTChunk = 32;                        // tokens of an epilogue step
constexpr int kTBox = 16;                          // tokens per TMA store

// For four epilogue warps: the other projection's sums [token][feature], and the results as they leave.
struct GatedTokensStage {
    alignas(1024) uint8_t out[3][kTChunk * 128];   // h, g, u
    alignas(1024) float up[kTChunk][64];
};

struct GatedTokensSmem {
    alignas(1024) uint8_t ring[kTRing];
    GatedTokensStage stage[2];
    alignas(16) uint64_t full[kTMostStages];       // leader's copy is the live one
    uint64_t empty[kTMostStages];                  // both, via multicast commit
    uint64_t tmem_full[2];                         // both, via multicast commit
    uint64_t tmem_empty[2];                        // leader's copy is the live one
    uint32_t tmem_base;
    int abort_flag;
};

struct GatedTokensMaps {
    CUtensorMap w[2], x, out[3];                   // weights; h, gate, up
};

struct GatedTokensParams {
    int32_t tokens, features, K;
    int32_t tile_tokens;         // multiple of 16, up to 256
    int32_t tiles_n, tiles;      // tiles of tokens; all
    int32_t k_steps;
    int32_t stage_bytes, stages;
    int32_t act, keep;
};

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kTThreads, 1)
gated_tokens_kernel(const __grid_constant__ GatedTokensMaps maps, const __grid_constant__ GatedTokensParams p)
{
    extern __shared__ uint8_t smem_raw[];
    GatedTokensSmem& sm = *reinterpret_cast<GatedTokensSmem*>(smem_align_1024(smem_raw));
    const int warp = threadIdx.x >> 5;
    const int lane = lane_id();
    const uint32_t rank = cluster_ctarank();
    const int cluster_id = blockIdx.x >> 1;
    const int n_clusters = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        sm.abort_flag = 0;
        for (int s = 0; s < kTMostStages; ++s) {
            mbar_init(&sm.full[s], 2);                 // one arrive.expect_tx per CTA
            mbar_init(&sm.empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&sm.tmem_full[b], 1);
            mbar_init(&sm.tmem_empty[b], 2 * 8);
        }
        fence_barrier_init();
    }
    if (warp == kTMmaWarp) {
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

    if (warp == kTProducerWarp) {
        // ------------------------------------------------------------ TMA producer
        if (elect_one_sync()) {
            int s = 0;
            uint32_t parity = 1;                       // of the phase before: a fresh barrier passes
            bool alive = true;
            const uint32_t bytes = kTWeightBytes + p.tile_tokens / 2 * 128;
            // the weights go past the tokens, which every tile reads
            const uint64_t kept = l2_policy_evict_last(), passing = l2_policy_evict_first();
            for (int tile = cluster_id; alive && tile < p.tiles; tile += n_clusters) {
                const int tm = tile / p.tiles_n, tn = tile - tm * p.tiles_n;
                const int f = tm * kTFeatures + static_cast<int>(rank) * 64;
                const int t = tn * p.tile_tokens + static_cast<int>(rank) * (p.tile_tokens / 2);
                for (int k = 0; k < p.k_steps; ++k) {
                    if (!mbar_wait(&sm.empty[s], parity, &sm.abort_flag)) {
                        alive = false;
                        break;
                    }
                    uint8_t* to = sm.ring + s * p.stage_bytes;
                    const uint32_t full = map_to_cta(smem_u32(&sm.full[s]), 0);
                    mbar_arrive_expect_tx_cluster(full, bytes);
                    tma_load_2d_pair_hint(to, &maps.w[0], full, k * kTBlockK, f, passing);
                    tma_load_2d_pair_hint(to + kTWeightBytes / 2, &maps.w[1], full, k * kTBlockK, f, passing);
                    tma_load_2d_pair_hint(to + kTWeightBytes, &maps.x, full, k * kTBlockK, t, kept);
                    if (++s == p.stages) {
                        s = 0;
                        parity ^= 1;
                    }
                }
            }
            // the last stages' release signals: one that arrived after the CTA is gone would be counted on a barrier
            // of the next launch
            for (int i = 0; alive && i < p.stages; ++i) {
                alive = mbar_wait(&sm.empty[s], parity, &sm.abort_flag);
                if (++s == p.stages) {
                    s = 0;
                    parity ^= 1;
                }
            }
            if (!alive) linger();      // given up: what is in flight lands before the CTA leaves
        }
        __syncwarp();
    } else if (warp == kTMmaWarp) {
        // ------------------------------------------------------------ MMA issuer
        if (rank == 0 && elect_one_sync()) {
            // fp32 accumulator, bf16 x bf16, 256 x tokens x 16, both along K
            const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(p.tile_tokens >> 3) << 17) |
                                   (static_cast<uint32_t>(256 >> 4) << 24);
            const uint64_t desc0 = make_smem_desc(smem_u32(sm.ring), 16, 1024, 2);
            int s = 0, b = 0;
            uint32_t parity = 0, buf_parity = 1;       // a fresh tmem_empty passes for the phase before
            bool alive = true;
            for (int tile = cluster_id; alive && tile < p.tiles; tile += n_clusters) {
                if (!mbar_wait(&sm.tmem_empty[b], buf_parity, &sm.abort_flag)) break;
                tcgen05_fence_after();
                for (int k = 0; k < p.k_steps; ++k) {
                    if (!mbar_wait(&sm.full[s], parity, &sm.abort_flag)) {
                        alive = false;
                        break;
                    }
                    tcgen05_fence_after();
                    const int nmma = (min(kTBlockK, p.K - k * kTBlockK) + 15) / 16;      // what lies past K is filled with zeros
                    const uint64_t a_desc = desc0 + static_cast<uint64_t>(s * (p.stage_bytes >> 4));
                    const uint64_t b_desc = a_desc + (kTWeightBytes >> 4);
#pragma unroll
                    for (int j = 0; j < kTBlockK / 16; ++j)
                        if (j < nmma) tcgen05_mma_f16_pair(tmem + b * 256, a_desc + 2 * j, b_desc + 2 * j, idesc, (k | j) > 0);
                    tcgen05_commit_pair(&sm.empty[s], 3);
                    if (++s == p.stages) {
                        s = 0;
                        parity ^= 1;
                    }
                }
                if (alive) tcgen05_commit_pair(&sm.tmem_full[b], 3);
                buf_parity ^= b;
                b ^= 1;
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------ epilogue warps
        const int quad = warp & 3;                     // TMEM lane quadrant of this warp: 0, 1 gate, 2, 3 the other projection
        const int half = warp >> 2;                    // even or odd chunks
        const bool gate = quad < 2;
        const int feature = (quad & 1) * 32 + lane;    // of the CTA's 64
        GatedTokensStage& st = sm.stage[half];
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        const uint32_t tmem_empty_leader = map_to_cta(smem_u32(&sm.tmem_empty[0]), 0);
        // a result's place in its staged row (128-byte swizzle)
        auto put = [&](int which, int token, float v) {
            uint8_t* row = st.out[which] + token * 128;
            smem_store(row + (((feature >> 3) ^ (token & 7)) * 16) + (feature & 7) * 2, __float2bfloat16_rn(v), st.out, sizeof(st.out));
        };
        int b = 0;
        uint32_t parity = 0;
        bool alive = true;
        for (int tile = cluster_id; tile < p.tiles; tile += n_clusters) {
            const int tm = tile / p.tiles_n, tn = tile - tm * p.tiles_n;
            const int f0 = tm * kTFeatures + static_cast<int>(rank) * 64;
            const int t0 = tn * p.tile_tokens;
            const int n = min(p.tile_tokens, p.tokens - t0);
            // given up: nothing more is stored, but the warps go on meeting at their barriers
            alive = mbar_wait(&sm.tmem_full[b], parity, &sm.abort_flag) && alive;
            tcgen05_fence_after();
            for (int c = half * kTChunk; c < n && f0 < p.features; c += 2 * kTChunk) {
                uint32_t r[32];
                tmem_ld_32x32b_x32(lanes + b * 256 + c, r);
                // the staged rows of the chunk before have left
                if (quad == 0 && lane == 0) bulk_wait_group_read<0>();
                bar_sync(1 + half, 128);
                tmem_ld_wait_for(r);
                if (!gate) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        smem_store(&st.up[i][feature], __uint_as_float(r[i]), st.up, sizeof(st.up));
                        if (p.keep) put(2, i, __uint_as_float(r[i]));
                    }
                }
                bar_sync(1 + half, 128);
                if (gate) {
                    if (p.keep) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) put(1, i, __uint_as_float(r[i]));
                    }
                    with_act(p.act, [&](auto act) {
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            put(0, i, act_value<decltype(act)::value>(__uint_as_float(r[i])) * smem_load<float>(&st.up[i][feature], st.up, sizeof(st.up)));
                    });
                }
                fence_proxy_async_smem();
                bar_sync(1 + half, 128);
                if (quad == 0 && lane == 0 && alive) {
                    for (int o = 0; o < (p.keep ? 3 : 1); ++o)
                        for (int i = 0; i < kTChunk && c + i < n; i += kTBox)
                            tma_store_2d(&maps.out[o], st.out[o] + i * 128, f0, t0 + c + i);
                    bulk_commit_group();
                }
            }
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(tmem_empty_leader + b * 8);
            parity ^= b;
            b ^= 1;
        }
        if (quad == 0 && lane == 0) bulk_wait_group<0>();
    }

    // neither CTA may leave (or free TMEM) while its peer can still signal it or read its memory
    tcgen05_fence_before();
    __syncthreads();
    cluster_sync_all();
    if (warp == kTMmaWarp) {
        tcgen05_fence_after();
        tmem_dealloc_pair(tmem, 512);
    }
}

}  // namespace mxfp4
