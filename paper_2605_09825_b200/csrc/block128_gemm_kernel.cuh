// 8-bit product with one fp32 scale per 128 elements along K:
//
//   out[m][n] = sum_t sa[t][m] * sb[t][n or n / 128] * sum_{k in block t} A[m][k] * B[n][k]
//
// CTA-pair kernel (tcgen05 cta_group::2) on 256 x 256 output tiles.  The scales are not powers of two, so the
// tensor cores cannot apply them: each K-step of 128 elements is a product of its own, formed in one
// of two TMEM buffers (2 x 256 columns: all of TMEM) while the epilogue warps read the other one and add
// it, scaled, to sums they keep in registers -- 128 rows x 256 columns per CTA, 128 sums per thread.
// Four K = 32 instructions are the longest chain of the tensor cores' truncating additions.  The two column
// halves of a buffer are handed over separately, each by a warp of its own: the four warps that read one
// half signal the issuer of that half.
//
// Per SM and K-step: 512 cycles of MMA; 128 x 256 multiply-adds of the epilogue, packed in pairs, are 256
// cycles of the FMA pipe (twice that when B has a scale per row, which costs a multiplication per
// element more).  Neither bounds the kernel (8192 x 28672 x 4096 by itself: 848 us, 2.3 PFLOP/s, 1.9 back to back, where the
// power cap holds 1.5 GHz; 28672 x 4096 x 8192 with a scale per row of B: 1202 us, 1.6, and 1.45 back to back at
// 1.64 GHz; 4096 x 4096 x 4096 with its join: 82 and 115 us.  A K-step takes 900 to 1000 cycles, 1400 with scales per
// row): a half buffer's way round does -- 256 cycles of MMA, about 200 until the epilogue has seen
// the signal, 500 to 700 of reading and adding (two warps per scheduler, which is what 128 sums per
// thread leave room for, cover little of each other's waits), 340 for the signal back across the pair,
// 100 to issue -- with two K-steps of tensor memory to overlap it.  With the additions left out it runs
// at 2.5-2.65 PFLOP/s.  Measured instead: one issuer for whole buffers (2.15), one issuer for both halves
// (1.85: its waits and commits become the chain), 256 x 192 tiles with five units of 96 columns in tensor
// memory and all 96 read ahead (1.63), both register sets loaded before each wait (1.7), scales fetched
// by the epilogue warps from global memory (2.1), the next scale fetched a K-step ahead (2.1; 1.5 instead
// of 1.7 with scales per row).
//
// Roles per CTA (384 threads): warps 0..7 epilogue (32 rows x 128 columns each), warp 8 TMA producer,
// warps 9 and 10 MMA issuers, one per column half (leader CTA only).  Barrier ownership as in the
// block-scaled kernel: full and tmem_empty live in the leader, empty and tmem_full are signalled in both
// CTAs by a multicast commit.  All waits are bounded.
//
// The output tiles that do not fill a wave of the 74 pairs -- all of them in a small product, the last ones in
// a large one -- are split along K where two or more pieces of each fit the wave: every piece writes its
// fp32 sums to the workspace, and a second kernel adds them in a fixed order.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>

#include <type_traits>

#include "../../include/mxfp4.h"
#include "ptx_sm100.cuh"
#include "row_io.cuh"
#include "tma_host.cuh"

namespace mxfp4 {

constexpr int kBTile = 256;                       // both ways
constexpr int kBHalf = 128;                       // rows of A, and of B, per CTA
constexpr int kBBlockK = 128;                     // elements = bytes per stage and row
constexpr int kBStages = 5;
constexpr int kBGroup = 4;                        // K-steps whose scales travel together
constexpr int kBGroups = 3;
constexpr int kBOperandBytes = kBHalf * kBBlockK; // 16 KB
constexpr int kBEpiWarps = 8;
constexpr int kBProducerWarp = 8;
constexpr int kBMmaWarp = 9;
constexpr int kBThreads = 384;
constexpr int kBStageBytes = 32 * 128;            // output staging per epilogue warp

struct Gemm128Smem {
    alignas(1024) uint8_t a[kBStages][kBOperandBytes];
    alignas(1024) uint8_t b[kBStages][2][kBOperandBytes / 2];   // [column half][64 rows x 128 B]
    alignas(1024) uint8_t out_stage[kBEpiWarps][kBStageBytes];
    alignas(128) float sa[kBGroups][kBGroup][kBHalf];     // scales of this CTA's rows
    alignas(128) float sb[kBGroups][kBGroup][kBTile];     // of the tile's columns; of its two blocks (128 x 128)
    alignas(32) uint64_t tmem_full[2][2];         // [column half][buffer]: both, via multicast commit
    alignas(32) uint64_t tmem_empty[2][2];        // leader's copy is the live one
    alignas(8) uint64_t full[kBStages];           // leader's copy is the live one
    uint64_t empty[kBStages];                     // both, via multicast commit
    uint64_t scales_full[kBGroups];               // local
    uint64_t scales_empty[kBGroups];              // local
    uint32_t tmem_base;
    int abort_flag;
};

struct Gemm128Params {
    const float* a_scales;
    const float* b_scales;
    void* out;                   // for the columns past the last 16-byte granule
    int64_t ld_out;
    int64_t pitch_a;             // scales per K-step of A, of B
    int64_t pitch_b;
    int32_t M, N, K;
    int32_t tiles_m, tiles_n;
    int32_t band;                // tile columns per band of the tile order
    int32_t k_steps;             // ceil(K / 128)
    int32_t whole;               // tiles with one piece; the others have `splits` along K
    int32_t splits;
    int32_t items;               // pieces of all tiles
    int32_t n_tma;               // columns written by TMA stores
};

// A piece of work: one output tile, one range of K-steps.  Tiles are numbered band by band: a band is
// `band` tile columns, sized so that its B panel stays in L2, and inside a band the tile column varies
// fastest, so that the tiles in flight share A rows and B columns.
struct Gemm128Work {
    int tm, tn, slot, k0, k1;    // slot: place of the sums in the workspace; -1: they are the output
};

// Row and column of a tile, counted in tiles.
__host__ __device__ __forceinline__ void gemm128_place(int tile, int band, int tiles_m, int tiles_n, int& tm, int& tn)
{
    const int per_band = band * tiles_m;
    const int b = tile / per_band;
    const int r = tile - b * per_band;
    const int cols = min(band, tiles_n - b * band);
    tm = r / cols;
    tn = b * band + (r - tm * cols);
}

__device__ __forceinline__ Gemm128Work gemm128_work(const Gemm128Params& p, int item)
{
    Gemm128Work w;
    int tile = item;
    w.slot = item - p.whole;
    w.k0 = 0;
    w.k1 = p.k_steps;
    if (w.slot < 0) {
        w.slot = -1;
    } else {
        const int t = w.slot / p.splits, split = w.slot - t * p.splits;
        tile = p.whole + t;
        w.k0 = static_cast<int>(static_cast<int64_t>(p.k_steps) * split / p.splits);
        w.k1 = static_cast<int>(static_cast<int64_t>(p.k_steps) * (split + 1) / p.splits);
    }
    gemm128_place(tile, p.band, p.tiles_m, p.tiles_n, w.tm, w.tn);
    return w;
}

// Columns the MMAs of a column half compute: what exists, rounded up to the instruction's granule (0: none).
// CTA r of the pair supplies rows [r * n / 2, (r + 1) * n / 2) of the half's n rows of B.
__device__ __forceinline__ int gemm128_width(int N, int tn, int half)
{
    return max(0, min(kBHalf, (N - tn * kBTile - half * kBHalf + 15) & ~15));
}

// BROWS: B has a scale per row and K-step (1 x 128 blocks); otherwise one per 128 rows.
template <bool BROWS, bool OUT32>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kBThreads, 1)
gemm_block128_pair_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b,
                          const __grid_constant__ CUtensorMap tm_out, const __grid_constant__ CUtensorMap tm_parts,
                          const Gemm128Params p)
{
    extern __shared__ uint8_t smem_raw[];
    Gemm128Smem& sm = *reinterpret_cast<Gemm128Smem*>(smem_align_1024(smem_raw));
    const int warp = threadIdx.x >> 5;
    const int lane = lane_id();
    const uint32_t rank = cluster_ctarank();
    const int cluster_id = blockIdx.x >> 1;
    const int n_clusters = gridDim.x >> 1;
    const int items = p.items;

    if (threadIdx.x == 0) {
        sm.abort_flag = 0;
        for (int s = 0; s < kBStages; ++s) {
            mbar_init(&sm.full[s], 2);                 // one arrive.expect_tx per CTA
            mbar_init(&sm.empty[s], 2);                // one commit per column half
        }
        for (int g = 0; g < kBGroups; ++g) {
            mbar_init(&sm.scales_full[g], BROWS ? 1 : 33);       // bulk copies; a word per lane of the producer
            mbar_init(&sm.scales_empty[g], kBEpiWarps);
        }
        for (int b = 0; b < 2; ++b) {
            for (int h = 0; h < 2; ++h) {
                mbar_init(&sm.tmem_full[h][b], 1);
                mbar_init(&sm.tmem_empty[h][b], kBEpiWarps);      // the half's four warps in each CTA
            }
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

    // registers: 384 x 168 at launch = 256 x 216 (epilogue) + 128 x 72 (the others)
    if (warp >= kBEpiWarps) {
        setmaxnreg_dec<72>();
        if (warp == kBProducerWarp) {
            // -------------------------------------------------------- TMA producer
            if (lane == 0) {
                tma_prefetch_desc(&tm_a);
                tma_prefetch_desc(&tm_b);
            }
            int s = 0, g = 0;
            uint32_t parity = 1, scale_parity = 1;     // of the phase before: a fresh barrier passes
            bool alive = true;
            for (int item = cluster_id; alive && item < items; item += n_clusters) {
                const Gemm128Work w = gemm128_work(p, item);
                const int32_t ya = w.tm * kBTile + static_cast<int>(rank) * kBHalf;
                // this CTA's share of each half's rows of B; the boxes are always 64 rows
                const int32_t yb0 = w.tn * kBTile + static_cast<int>(rank) * (gemm128_width(p.N, w.tn, 0) >> 1);
                const int32_t yb1 = w.tn * kBTile + kBHalf + static_cast<int>(rank) * (gemm128_width(p.N, w.tn, 1) >> 1);
                // scales: as far as the scale arrays reach (whole blocks of 128 rows); none for a CTA without rows, whose
                // epilogue warps wait for none (a copy nobody waits for may land after the CTA is gone)
                const bool rows = ya < p.M;
                const uint32_t a_bytes = rows ? kBHalf * 4 : 0;
                const uint32_t b_bytes =
                    BROWS && rows ? static_cast<uint32_t>(min(static_cast<int64_t>(kBTile), p.pitch_b - w.tn * kBTile)) * 4
                                  : 0;
                for (int k = w.k0; k < w.k1; ++k) {
                    const bool group = ((k - w.k0) & (kBGroup - 1)) == 0;
                    if (!mbar_wait(&sm.empty[s], parity, &sm.abort_flag) ||
                        (group && !mbar_wait(&sm.scales_empty[g], scale_parity, &sm.abort_flag))) {
                        alive = false;
                        break;
                    }
                    if (elect_one_sync()) {
                        const uint32_t full_leader = map_to_cta(smem_u32(&sm.full[s]), 0);
                        mbar_arrive_expect_tx_cluster(full_leader, 2 * kBOperandBytes);
                        tma_load_2d_pair(sm.a[s], &tm_a, full_leader, k * kBBlockK, ya);
                        tma_load_2d_pair(sm.b[s][0], &tm_b, full_leader, k * kBBlockK, yb0);
                        tma_load_2d_pair(sm.b[s][1], &tm_b, full_leader, k * kBBlockK, yb1);
                        if (group) {
                            const int n = min(kBGroup, w.k1 - k);
                            mbar_arrive_expect_tx(&sm.scales_full[g], n * (a_bytes + b_bytes));
                            for (int i = 0; i < n; ++i) {
                                if (a_bytes)
                                    bulk_load_1d(sm.sa[g][i], p.a_scales + (k + i) * p.pitch_a + ya, a_bytes,
                                                 &sm.scales_full[g]);
                                if (b_bytes)
                                    bulk_load_1d(sm.sb[g][i], p.b_scales + (k + i) * p.pitch_b + w.tn * kBTile, b_bytes,
                                                 &sm.scales_full[g]);
                            }
                        }
                    }
                    __syncwarp();
                    if (!BROWS && group) {
                        // the tile's columns are two blocks of 128: two words per K-step, one per lane
                        const int i = lane >> 1, block = 2 * w.tn + (lane & 1);
                        if (rows && i < min(kBGroup, w.k1 - k) && block < p.pitch_b && smem_within(sm.sb[g], i))
                            cp_async_word(&sm.sb[g][i][lane & 1], p.b_scales + (k + i) * p.pitch_b + block);
                        cp_async_arrive(&sm.scales_full[g]);
                    }
                    if (++s == kBStages) {
                        s = 0;
                        parity ^= 1;
                    }
                    if (group && ++g == kBGroups) {
                        g = 0;
                        scale_parity ^= 1;
                    }
                }
            }
            // the last stages' release signals: one that arrived after the CTA is gone would be counted on a barrier
            // of the next launch
            for (int i = 0; alive && i < kBStages; ++i) {
                alive = mbar_wait(&sm.empty[s], parity, &sm.abort_flag);
                if (++s == kBStages) {
                    s = 0;
                    parity ^= 1;
                }
            }
            if (!alive) linger();      // given up: what is in flight lands before the CTA leaves
        } else if (warp < kBMmaWarp + 2 && rank == 0) {
            // -------------------------------------------------------- MMA issuers, one per column half
            const int half = warp - kBMmaWarp;
            const uint64_t a_desc0 = make_smem_desc(smem_u32(sm.a[0]), 16, 1024, 2);
            const uint64_t b_desc0 = make_smem_desc(smem_u32(sm.b[0][half]), 16, 1024, 2);
            const uint32_t full = smem_u32(&sm.full[0]), tmem_empty = smem_u32(&sm.tmem_empty[half][0]);
            int s = 0, b = 0;
            uint32_t parity = 0, buf_parity = 1;       // a fresh tmem_empty passes for the phase before
            bool alive = true;
            for (int item = cluster_id; alive && item < items; item += n_clusters) {
                const Gemm128Work w = gemm128_work(p, item);
                const int width = gemm128_width(p.N, w.tn, half);
                // instruction descriptor: fp32 accumulator, E4M3 x E4M3, K-major operands
                const uint32_t idesc = (1u << 4) | (static_cast<uint32_t>(width >> 3) << 17) |
                                       (static_cast<uint32_t>(kBTile >> 4) << 24);
                for (int k = w.k0; k < w.k1; ++k) {
                    if (!mbar_wait_addr(full + s * 8, parity, &sm.abort_flag) ||
                        !mbar_wait_addr(tmem_empty + b * 8, buf_parity, &sm.abort_flag)) {
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
                            if (j < nmma && width > 0)
                                tcgen05_mma_f8_pair(tmem + b * kBTile + half * kBHalf, a_desc + 2 * j, b_desc + 2 * j, idesc,
                                                    j > 0);
                        tcgen05_commit_pair(&sm.empty[s], 3);
                        tcgen05_commit_pair(&sm.tmem_full[half][b], 3);
                    }
                    __syncwarp();
                    if (++s == kBStages) {
                        s = 0;
                        parity ^= 1;
                    }
                    buf_parity ^= b;
                    b ^= 1;
                }
            }
        }
    } else {
        // ------------------------------------------------------------ epilogue warps
        setmaxnreg_inc<216>();
        const int quad = warp & 3;                     // TMEM lane quadrant of this warp
        const int half = warp >> 2;                    // which 128 columns
        uint8_t* stg = sm.out_stage[warp];
        const uint32_t taddr0 = tmem + (static_cast<uint32_t>(quad * 32) << 16) + half * kBHalf;
        const uint32_t tmem_empty_leader = map_to_cta(smem_u32(&sm.tmem_empty[half][0]), 0);
        // the buffer at hand: its columns, its barriers, the parity of its phase
        uint32_t buf = 0, from = taddr0, parity = 0;
        uint32_t full = smem_u32(&sm.tmem_full[half][0]), empty = tmem_empty_leader;
        auto next_buffer = [&]() {
            from ^= kBTile;                            // the two buffers start at a multiple of 512 columns
            full ^= 8;                                 // two barriers, aligned to both
            empty ^= 8;
            parity ^= buf;
            buf ^= 1;
        };
        int g = 0;                                     // scale group at hand
        uint32_t scale_parity = 0;
        auto release_group = [&]() {
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.scales_empty[g]);
            if (++g == kBGroups) {
                g = 0;
                scale_parity ^= 1;
            }
        };
        bool alive = true;
        for (int item = cluster_id; alive && item < items; item += n_clusters) {
            const Gemm128Work w = gemm128_work(p, item);
            const int row0 = w.tm * kBTile + static_cast<int>(rank) * kBHalf + quad * 32;
            const int col0 = w.tn * kBTile + half * kBHalf;
            const bool row_ok = row0 + lane < p.M;
            if (row0 >= p.M || col0 >= p.N) {          // warp-uniform: nothing to keep here
                for (int k = w.k0; alive && k < w.k1; ++k) {
                    alive = mbar_wait_addr(full, parity, &sm.abort_flag);
                    if (lane == 0) mbar_arrive_cluster(empty);
                    next_buffer();
                    if (((k - w.k0) & (kBGroup - 1)) == kBGroup - 1 || k + 1 == w.k1) release_group();
                }
                continue;
            }
            float2 acc[64];
#pragma unroll
            for (int i = 0; i < 64; ++i) acc[i] = make_float2(0.0f, 0.0f);
            // a K-step's scale of this thread's row (times the one of the 128 columns)
            auto scale_of = [&](int in_group) {
                float v = smem_load<float>(sm.sa[g][in_group] + quad * 32 + lane, sm.sa[g], sizeof(sm.sa[0]));
                if (!BROWS) v *= smem_load<float>(sm.sb[g][in_group] + half, sm.sb[g], sizeof(sm.sb[0]));
                return v;
            };
            alive = mbar_wait(&sm.scales_full[g], scale_parity, &sm.abort_flag);
            float scale = scale_of(0);
            uint32_t r0[32], r1[BROWS ? 1 : 32];
            bool started = false;
            for (int k = w.k0; k < w.k1; ++k) {
                const int in_group = (k - w.k0) & (kBGroup - 1);
                const bool more = k + 1 < w.k1;
                const float* sb = sm.sb[g][in_group] + half * kBHalf;
                const float2 scale2 = make_float2(scale, scale);
                if (!started) {
                    alive = mbar_wait_addr(full, parity, &sm.abort_flag) && alive;
                    tcgen05_fence_after();
                    if (!BROWS) tmem_ld_32x32b_x32(from, r0);
                }
                auto hand_back = [&]() {
                    tcgen05_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(empty);
                    next_buffer();
                };
                if constexpr (BROWS) {
                    // a chunk's products and its columns' scales arrive together, while the other warp of the scheduler
                    // works on its chunk
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        tmem_ld_32x32b_x32(from + c * 32, r0);
                        float4 e[4];                   // column scales, sixteen at a time
                        auto load_scales = [&](float4 (&to)[4], int i0) {
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                to[i] = smem_load<float4>(sb + c * 32 + (i0 + i) * 4, sb, kBHalf * 4);
                        };
                        auto add = [&](const float4 (&e)[4], int i0) {
#pragma unroll
                            for (int i = i0; i < i0 + 4; ++i) {
                                const float4& f = e[i - i0];
                                const float2 v0 = __fmul2_rn(
                                    make_float2(__uint_as_float(r0[4 * i]), __uint_as_float(r0[4 * i + 1])), make_float2(f.x, f.y));
                                const float2 v1 = __fmul2_rn(
                                    make_float2(__uint_as_float(r0[4 * i + 2]), __uint_as_float(r0[4 * i + 3])), make_float2(f.z, f.w));
                                acc[c * 16 + 2 * i] = __ffma2_rn(v0, scale2, acc[c * 16 + 2 * i]);
                                acc[c * 16 + 2 * i + 1] = __ffma2_rn(v1, scale2, acc[c * 16 + 2 * i + 1]);
                            }
                        };
                        load_scales(e, 0);
                        tmem_ld_wait_for(r0);
                        if (c == 3) hand_back();
                        add(e, 0);
                        load_scales(e, 4);
                        add(e, 4);
                    }
                } else {
                    // two register sets take turns: while one chunk of 32 columns is scaled and added, the next one is on
                    // its way from tensor memory, across K-steps too where the next product is ready in time
                    auto add = [&](int c, const uint32_t (&r)[32]) {
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            acc[c * 16 + i] = __ffma2_rn(make_float2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1])),
                                                         scale2, acc[c * 16 + i]);
                    };
                    tmem_ld_wait_for(r0);
                    tmem_ld_32x32b_x32(from + 32, r1);
                    add(0, r0);
                    tmem_ld_wait_for(r1);
                    tmem_ld_32x32b_x32(from + 64, r0);
                    add(1, r1);
                    tmem_ld_wait_for(r0);
                    tmem_ld_32x32b_x32(from + 96, r1);
                    add(2, r0);
                    tmem_ld_wait_for(r1);
                    hand_back();
                    started = more && __all_sync(0xffffffffu, mbar_test_wait_addr(full, parity));
                    if (started) {
                        tcgen05_fence_after();
                        tmem_ld_32x32b_x32(from, r0);
                    }
                    add(3, r1);
                }
                if (in_group == kBGroup - 1 || !more) {
                    release_group();
                    if (more) alive = mbar_wait(&sm.scales_full[g], scale_parity, &sm.abort_flag) && alive;
                }
                if (more) scale = scale_of((in_group + 1) & (kBGroup - 1));
            }
            if (!alive) break;                         // a wait was given up: nothing of this tile is stored
            // the warp's 32 rows x 128 columns leave in boxes of 128 bytes per row, staged in the 128-byte
            // swizzle for a TMA store that clips at the matrix edges
            auto stage_box = [&](auto fp32, int c) {
                if (lane == 0) bulk_wait_group_read<0>();
                __syncwarp();
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    uint8_t* to = stg + lane * 128 + ((q ^ (lane & 7)) * 16);
                    if constexpr (decltype(fp32)::value) {
                        // two words at a time: four would have to sit in adjacent registers, which the sums' pairs do not
                        smem_store(to, acc[c * 16 + 2 * q], stg, kBStageBytes);
                        smem_store(to + 8, acc[c * 16 + 2 * q + 1], stg, kBStageBytes);
                    } else {
                        const float2* x = &acc[c * 32 + 4 * q];
                        smem_store(to, make_uint4(pack_bf16(x[0].x, x[0].y), pack_bf16(x[1].x, x[1].y),
                                                  pack_bf16(x[2].x, x[2].y), pack_bf16(x[3].x, x[3].y)), stg, kBStageBytes);
                    }
                }
                fence_proxy_async_smem();
                __syncwarp();
            };
            if (w.slot >= 0) {
                // a piece of a tile: its sums have a place of their own in the workspace
#pragma unroll
                for (int c = 0; c < kBHalf / 32; ++c) {
                    stage_box(std::true_type{}, c);
                    if (lane == 0) {
                        tma_store_3d(&tm_parts, stg, half * kBHalf + c * 32, static_cast<int>(rank) * kBHalf + quad * 32,
                                     w.slot);
                        bulk_commit_group();
                    }
                }
                continue;
            }
            constexpr int kBoxCols = OUT32 ? 32 : 64;
            constexpr int kGranule = OUT32 ? 4 : 8;
#pragma unroll
            for (int c = 0; c < kBHalf / kBoxCols; ++c) {
                const int col = col0 + c * kBoxCols;
                stage_box(std::bool_constant<OUT32>{}, c);
                // columns past the last full 16-byte granule, one by one from the staged row
                const int rc = p.n_tma - col;
                if (p.n_tma < p.N && rc >= 0 && rc < kBoxCols && row_ok) {
                    const int q = rc / kGranule;
                    const uint4 v = smem_load<uint4>(stg + lane * 128 + ((q ^ (lane & 7)) * 16), stg, kBStageBytes);
                    const int64_t at = static_cast<int64_t>(row0 + lane) * p.ld_out + p.n_tma;
                    const uint32_t e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int j = 0; j < kGranule; ++j)
                        if (p.n_tma + j < p.N) {
                            if (OUT32) static_cast<uint32_t*>(p.out)[at + j] = e[j & 3];
                            else static_cast<uint16_t*>(p.out)[at + j] = static_cast<uint16_t>(e[j >> 1] >> (16 * (j & 1)));
                        }
                }
                if (lane == 0 && col < p.n_tma) {
                    tma_store_3d(&tm_out, stg, col, row0, 0);
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

// Sum of the pieces of the split tiles, in their order; four columns per thread.
struct Gemm128JoinParams {
    const float* parts;          // [split tile][piece][rows][256]
    void* out;
    int64_t ld_out;
    int32_t M, N;
    int32_t whole;               // the first split tile
    int32_t splits;
    int32_t rows;                // min(M, 256)
    int32_t band, tiles_m, tiles_n;
    int32_t out_fp32;
};

constexpr int kBJoinRows = 4;    // per block, four columns per thread

__global__ void __launch_bounds__(256) gemm_block128_join_kernel(const Gemm128JoinParams p)
{
    griddep_launch_dependents();
    const int per_tile = (p.rows + kBJoinRows - 1) / kBJoinRows;
    const int t = blockIdx.x / per_tile;
    const int r = (blockIdx.x - t * per_tile) * kBJoinRows + threadIdx.x / (kBTile / 4);
    const int c = threadIdx.x % (kBTile / 4) * 4;
    int tm, tn;
    gemm128_place(p.whole + t, p.band, p.tiles_m, p.tiles_n, tm, tn);
    const int64_t row = static_cast<int64_t>(tm) * kBTile + r;
    const int64_t col = static_cast<int64_t>(tn) * kBTile + c;
    if (r >= p.rows || row >= p.M || col >= p.N) return;
    griddep_wait();
    const int64_t piece = static_cast<int64_t>(p.rows) * kBTile;
    const float* from = p.parts + t * p.splits * piece + r * kBTile + c;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int i = 0; i < p.splits; ++i) {
        const float4 v = *reinterpret_cast<const float4*>(from + i * piece);
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    const float e[4] = {s.x, s.y, s.z, s.w};
    if (col + 3 < p.N) {                                     // rows start at multiples of 16 bytes
        if (p.out_fp32) *reinterpret_cast<float4*>(static_cast<float*>(p.out) + row * p.ld_out + col) = s;
        else *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + row * p.ld_out + col) =
            make_uint2(pack_bf16(s.x, s.y), pack_bf16(s.z, s.w));
        return;
    }
#pragma unroll
    for (int j = 0; j < 3; ++j)
        if (col + j < p.N) {
            if (p.out_fp32) static_cast<float*>(p.out)[row * p.ld_out + col + j] = e[j];
            else static_cast<__nv_bfloat16*>(p.out)[row * p.ld_out + col + j] = __float2bfloat16_rn(e[j]);
        }
}

}  // namespace mxfp4
