// Product of 16-bit matrices with a fused epilogue: D[m][n] = sum_k A[m][k] * B[n][k], fp32 sums in tensor memory.
//
// CTA-pair kernel (tcgen05 cta_group::2, kind::f16) on 256 x 256 output tiles: each CTA holds 128 rows of A and 128
// rows of B per K-step of 64 elements (32 KB), five or six steps in flight, two accumulators of 256 columns (all of
// tensor memory), so that the epilogue of one tile runs under the products of the next.  A step takes 512 cycles of the
// tensor cores and as many of the way from L2 into shared memory (64 bytes per cycle and SM): a larger tile would need more
// tensor memory.  The tensor pipe is busy 91 % of the cycles in the loss's forward product, 87 % in the gated one with both
// projections kept, 88 % in a backward pass; what it does per second is set by the power cap: 1.5 to 1.6 PFLOP/s for the
// loss of 8192 tokens by itself, 1.3 to 1.42 pass after pass (a library product: 1.69 and 1.39).
//
// Either operand may be stored along K (rows of A, of B) or along its own rows (the transposed matrix, as the
// gradients need it): a K-step is then fetched as two boxes of 64 columns x 64 rows, and the shared-memory
// descriptor names the transposed layout.  No transposed copy exists anywhere.
//
// Two matrices of the same shape may stand in for one along M (both weight gradients of a pair of projections in
// one launch) or along K (the input's gradient, a sum of two products).  A launch may take two products: tiles of the
// second fill the pairs that a last round of the first leaves idle, as many as one of the first's is long.  A
// product of few tiles is split along K, each piece with an output of its own, which the caller adds up.
//
// Epilogues:
//   kDenseStore             the sums, rounded or not, or added to the fp32 output by the copy engine: one addition per element
//                           and launch, so results do not depend on scheduling
//   kDenseScaled            the same of sums multiplied by a common factor (dense_common)
//   kDenseGated             columns 0..127 of a tile are a gate's, 128..255 the other projection's of the same features
//                           (the pair's first CTA loads the rows of one weight, the second those of the other): act(g) * u,
//                           and g and u on request
//   kDensePartials          maximum and sum of exponentials of each row's 128 columns, and the target's value.  The normaliser
//                           goes by a row's largest logits, and truncating additions make these too small, all alike: sums of
//                           4096 products left lse 1.9e-6 of itself off, sums of 1024, added in registers, 0.4e-6, at no cost
//   kDenseLogitGrad         gradient of the log probabilities with respect to the logits, without the factor that the
//                           positions have in common, rounded to bf16
//
// Roles per CTA (384 threads): warps 0..7 epilogue (32 rows x 128 columns each), warp 8 TMA producer, warp 9 MMA
// issuer (leader CTA only).  Barrier ownership: full and tmem_empty live in the leader, empty and tmem_full are signalled
// in both CTAs by a multicast commit.  All waits are bounded.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>

#include <type_traits>

#include "../../include/mxfp4.h"
#include "activations.cuh"
#include "dense_gemm.cuh"
#include "ptx_sm100.cuh"
#include "row_io.cuh"

namespace mxfp4 {

constexpr int kDTile = 256;                        // both ways
constexpr int kDHalf = 128;                        // rows of A, and of B, per CTA
constexpr int kDBlockK = 64;                       // elements: 128 bytes
constexpr int kDOperandBytes = kDHalf * kDBlockK * 2;
constexpr int kDBoxBytes = kDOperandBytes / 2;     // 64 columns x 64 rows of a transposed operand
constexpr int kDEpiWarps = 8;
constexpr int kDProducerWarp = 8;
constexpr int kDMmaWarp = 9;
constexpr int kDThreads = 384;                      // two warps more than there are roles: registers go by four warps
constexpr int kDChain = 16;
constexpr int kDStageBytes = 32 * 128;             // output staging per epilogue warp and box

// Two output boxes per warp, so that one is filled while the other leaves, are worth a stage of operands where tiles are
// short: the backward pass of 64 tokens (4096 x 14336) took 147 us with them and 162 without.  The gated forward pass has
// long ones: 104 us for 333 tokens with six stages, 107 with five and two boxes (before that size went to another kernel).
template <int EPI>
struct DenseSmem {
    static constexpr int kBoxes = EPI == kDenseStore || EPI == kDenseScaled ? 2 : 1;
    static constexpr int kDStages = 7 - kBoxes;
    alignas(1024) uint8_t a[kDStages][kDOperandBytes];
    alignas(1024) uint8_t b[kDStages][kDOperandBytes];
    alignas(1024) uint8_t out_stage[kDEpiWarps][kBoxes][kDStageBytes];
    alignas(16) uint64_t full[kDStages];           // leader's copy is the live one
    uint64_t empty[kDStages];                      // both, via multicast commit
    uint64_t tmem_full[2];                         // both, via multicast commit
    uint64_t tmem_empty[2];                        // leader's copy is the live one
    float2 common[kDEpiWarps];                     // of dense_common
    uint32_t tmem_base;
    int abort_flag;
};

struct DenseMaps {
    CUtensorMap a[2], b[2], out[3];
};
struct DenseMaps2 {
    DenseMaps q[2];              // of a launch's products
};

// A piece of work: a tile of one of the products, a range of K-steps of it.
struct DenseWork {
    int q;                       // product; -1: no more work
    int tm, tn;
    int seg;                     // segment along M
    int row;                     // first row of the tile, in its segment
    int out_row;                 // in the output
    int k0, k1;
};

// The j-th piece of work of a pair.  The first product's pieces go round the pairs; those that a last round leaves out take
// as many of the second product's as one of the first's is long, and the rest of these goes round all pairs,
// beginning with them.
template <bool TWO>
__device__ __forceinline__ DenseWork dense_work(const DenseParams& p, int pair, int pairs, int j)
{
    DenseWork w;
    int item = pair + j * pairs;
    w.q = 0;
    if (item >= p.q[0].items) {
        w.q = -1;
        if (!TWO || p.q[1].items == 0) return w;
        const int n0 = p.q[0].items, n1 = p.q[1].items;
        const int left = n0 % pairs;               // pairs that the first product's last round keeps busy
        const int idle = pairs - left;
        int extra = 0;                             // pieces of the second product for each of the others
        if (left > 0) {
            // a tile costs about eight steps besides its own
            extra = (p.q[0].k_steps / p.q[0].splits + 8) / (p.q[1].k_steps + 8);
            extra = min(extra, n1 / idle);
        }
        int i = j - n0 / pairs - (pair < left);
        if (pair >= left && i < extra) {
            item = pair - left + i * idle;
        } else {
            if (pair >= left) i -= extra;
            item = idle * extra + (pair >= left ? pair - left : pair + idle) + i * pairs;
        }
        if (item >= n1) return w;
        w.q = 1;
    }
    const DenseShape& q = p.q[w.q];
    // tiles band by band: a band is so many tile columns (or rows), and inside it they vary fastest, so that the tiles in
    // flight share rows of A and columns of B, and the band's panel stays in L2 while the other operand passes
    const int tiles = q.tiles_m * q.tiles_n;
    const int split = item / tiles, tile = item - split * tiles;
    const int across = q.band_m ? q.tiles_m : q.tiles_n, along = q.band_m ? q.tiles_n : q.tiles_m;
    const int per_band = q.band * along;
    const int b = tile / per_band;
    const int r = tile - b * per_band;
    const int wide = min(q.band, across - b * q.band);
    const int slow = r / wide, fast = b * q.band + (r - slow * wide);
    w.tm = q.band_m ? fast : slow;
    w.tn = q.band_m ? slow : fast;
    w.seg = w.tm >= q.seg_tiles_m;
    w.row = (w.tm - w.seg * q.seg_tiles_m) * kDTile;
    w.out_row = w.row + split * q.split_rows;
    w.k0 = static_cast<int>(static_cast<int64_t>(q.k_steps) * split / q.splits);
    w.k1 = static_cast<int>(static_cast<int64_t>(q.k_steps) * (split + 1) / q.splits);
    return w;
}

// One operand of a K-step: 128 rows x 64 elements of K, or the transposed 64 x 128 in two boxes.
__device__ __forceinline__ void dense_load(bool mn, uint8_t* to, const CUtensorMap* map, uint32_t bar, int row, int k, bool hint,
                                           uint64_t policy)
{
    const int x = mn ? row : k, y = mn ? k : row;
    if (hint) tma_load_2d_pair_hint(to, map, bar, x, y, policy);
    else tma_load_2d_pair(to, map, bar, x, y);
    if (mn) {
        if (hint) tma_load_2d_pair_hint(to + kDBoxBytes, map, bar, x + 64, y, policy);
        else tma_load_2d_pair(to + kDBoxBytes, map, bar, x + 64, y);
    }
}

// eight sums as bf16
__device__ __forceinline__ uint4 dense_pack8(const uint32_t* v)
{
    auto two = [&](int i) { return pack_bf16(__uint_as_float(v[i]), __uint_as_float(v[i + 1])); };
    return make_uint4(two(0), two(2), two(4), two(6));
}

// exp(x) of a difference to a maximum or a normaliser
__device__ __forceinline__ float dense_exp(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x * 1.4426950408889634f));
    return r;
}

// The factor that the gradients of all positions have in common, by which those of the logits are divided before they are
// rounded, and sums of them multiplied: the largest magnitude of d_logp at a target, so that the gradient of a mean is 1 or -1
// everywhere, unless d_lse is 2^60 times as large.  What is not finite is passed by.  The epilogue's warps find it while the
// first tile's products run; rounding the common factor with the rest would leave every result off by as much, up to
// 2^-8, all to the same side.  The multiplications show where tiles are one step long (loss backward of 64 tokens 617 -> 637 us,
// 512 tokens and more the same), so other products have an epilogue without them.
__device__ __forceinline__ float dense_common(const DenseExtra& x, float2 (&part)[kDEpiWarps], int warp, int lane)
{
    float2 most = make_float2(0.0f, 0.0f);
    auto take = [](float& m, float v) {
        v = fabsf(v);
        if (v <= 3.402823466e38f) m = fmaxf(m, v);
    };
#pragma unroll 8
    for (int64_t i = warp * 32 + lane; i < x.rows; i += kDEpiWarps * 32) {
        const int64_t target = x.d_logp ? x.targets[i] : -1;
        const float gl = x.d_logp ? x.d_logp[i] : 0.0f, gn = x.d_lse ? x.d_lse[i] : 0.0f;
        if (target >= 0) take(most.x, gl);
        take(most.y, gn);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        most.x = fmaxf(most.x, __shfl_xor_sync(0xffffffffu, most.x, d));
        most.y = fmaxf(most.y, __shfl_xor_sync(0xffffffffu, most.y, d));
    }
    if (lane == 0) smem_put(part, warp, most);
    bar_sync(1, kDEpiWarps * 32);
    for (int w = 0; w < kDEpiWarps; ++w) {
        const float2 v = smem_get(part, w);
        most = make_float2(fmaxf(most.x, v.x), fmaxf(most.y, v.y));
    }
    const float common = fmaxf(most.x, most.y * 0x1p-60f);
    return common > 0.0f ? common : 1.0f;
}

// kDenseStore and kDenseScaled take B along its own rows and two products; the other epilogues take both operands along K
// and one product.
template <int EPI>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kDThreads, 1)
dense_gemm_kernel(const __grid_constant__ DenseMaps2 maps, const __grid_constant__ DenseParams p)
{
    extern __shared__ uint8_t smem_raw[];
    DenseSmem<EPI>& sm = *reinterpret_cast<DenseSmem<EPI>*>(smem_align_1024(smem_raw));
    constexpr int kDStages = DenseSmem<EPI>::kDStages, kBoxes = DenseSmem<EPI>::kBoxes;
    const int warp = threadIdx.x >> 5;
    const int lane = lane_id();
    const uint32_t rank = cluster_ctarank();
    const int cluster_id = blockIdx.x >> 1;
    const int n_clusters = gridDim.x >> 1;
    constexpr bool kStore = EPI == kDenseStore || EPI == kDenseScaled;
    constexpr bool kGated = EPI == kDenseGated;
    // K-steps that are added up in tensor memory, whose additions truncate; longer sums go on in registers (0: any length)
    constexpr int kChain = EPI == kDensePartials ? kDChain : 0;

    if (threadIdx.x == 0) {
        sm.abort_flag = 0;
        for (int s = 0; s < kDStages; ++s) {
            mbar_init(&sm.full[s], 2);                 // one arrive.expect_tx per CTA
            mbar_init(&sm.empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&sm.tmem_full[b], 1);
            mbar_init(&sm.tmem_empty[b], 2 * kDEpiWarps);
        }
        fence_barrier_init();
    }
    if (warp == kDMmaWarp) {
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
    if (warp >= kDEpiWarps) {
        setmaxnreg_dec<72>();
        if (warp == kDProducerWarp) {
            // ------------------------------------------------------------ TMA producer
            if (elect_one_sync()) {
                int s = 0;
                uint32_t parity = 1;                       // of the phase before: a fresh barrier passes
                bool alive = true;
                const uint64_t kept = l2_policy_evict_last(), passing = l2_policy_evict_first();
                for (int j = 0; alive; ++j) {
                    const DenseWork w = dense_work<kStore>(p, cluster_id, n_clusters, j);
                    if (w.q < 0) break;
                    const DenseShape& q = p.q[w.q];
                    const DenseMaps& m = maps.q[w.q];
                    const bool a_mn = kStore && q.a_mn;
                    // without the hints where a launch holds two products: they bring nothing there (backward of 4096 tokens
                    // 1570 us either way), and issuing them costs where K is short (512 tokens: 188 us, 195 with them)
                    const bool hints = !kStore && q.hints;
                    const uint64_t pol_a = q.band_m ? kept : passing, pol_b = q.band_m ? passing : kept;
                    const int ya = w.row + static_cast<int>(rank) * kDHalf;
                    const int yb = kGated ? w.tn * q.width : w.tn * 2 * q.width + static_cast<int>(rank) * q.width;
                    for (int k = w.k0; k < w.k1; ++k) {
                        if (!mbar_wait(&sm.empty[s], parity, &sm.abort_flag)) {
                            alive = false;
                            break;
                        }
                        const int seg_k = k >= q.seg_k_steps;
                        const int kk = (k - seg_k * q.seg_k_steps) * kDBlockK;
                        const uint32_t full = map_to_cta(smem_u32(&sm.full[s]), 0);
                        mbar_arrive_expect_tx_cluster(full, kDOperandBytes + q.width * (kDBlockK * 2));
                        dense_load(a_mn, sm.a[s], &m.a[w.seg + seg_k], full, ya, kk, hints, pol_a);
                        dense_load(kStore, sm.b[s], &m.b[kGated ? rank : seg_k], full, yb, kk, hints, pol_b);
                        if (++s == kDStages) {
                            s = 0;
                            parity ^= 1;
                        }
                    }
                }
                // the last stages' release signals: one that arrived after the CTA is gone would be counted on a barrier
                // of the next launch
                for (int i = 0; alive && i < kDStages; ++i) {
                    alive = mbar_wait(&sm.empty[s], parity, &sm.abort_flag);
                    if (++s == kDStages) {
                        s = 0;
                        parity ^= 1;
                    }
                }
                if (!alive) linger();      // given up: what is in flight lands before the CTA leaves
            }
            __syncwarp();
        } else if (warp == kDMmaWarp) {
            // ------------------------------------------------------------ MMA issuer
            if (rank == 0 && elect_one_sync()) {
                // fp32 accumulator, bf16 x bf16, 256 x 2 * width x 16
                constexpr uint32_t idesc0 = (1u << 4) | (1u << 7) | (1u << 10) | (kStore ? 1u << 16 : 0u) |
                                            (static_cast<uint32_t>(kDTile >> 4) << 24);
                // along K: 8-row groups 1024 bytes apart, an instruction's 16 elements are 32 bytes; transposed: 64-column boxes
                // 8 KB apart, 8-row groups of K 1024 bytes apart, 16 rows are 2 KB
                const uint64_t b_desc0 = make_smem_desc(smem_u32(sm.b[0]), kStore ? kDBoxBytes : 16, 1024, 2);
                constexpr int kStepB = kStore ? 128 : 2;
                int s = 0, b = 0;
                uint32_t parity = 0, buf_parity = 1;       // a fresh tmem_empty passes for the phase before
                bool alive = true;
                for (int i = 0; alive; ++i) {
                    const DenseWork w = dense_work<kStore>(p, cluster_id, n_clusters, i);
                    if (w.q < 0) break;
                    const DenseShape& q = p.q[w.q];
                    const bool a_mn = kStore && q.a_mn;
                    const uint64_t a_desc0 = make_smem_desc(smem_u32(sm.a[0]), a_mn ? kDBoxBytes : 16, 1024, 2);
                    const int step_a = a_mn ? 128 : 2;
                    const uint32_t idesc = idesc0 | (a_mn ? 1u << 15 : 0u) | (static_cast<uint32_t>(2 * q.width) >> 3 << 17);
                    if (!mbar_wait(&sm.tmem_empty[b], buf_parity, &sm.abort_flag)) break;
                    tcgen05_fence_after();
                    int first = w.k0;                      // of the chain of additions
                    for (int k = w.k0; k < w.k1; ++k) {
                        if (kChain > 0 && k - first == kChain) {
                            tcgen05_commit_pair(&sm.tmem_full[b], 3);
                            buf_parity ^= b;
                            b ^= 1;
                            first = k;
                            if (!mbar_wait(&sm.tmem_empty[b], buf_parity, &sm.abort_flag)) {
                                alive = false;
                                break;
                            }
                            tcgen05_fence_after();
                        }
                        if (!mbar_wait(&sm.full[s], parity, &sm.abort_flag)) {
                            alive = false;
                            break;
                        }
                        tcgen05_fence_after();
                        const int kk = (k >= q.seg_k_steps ? k - q.seg_k_steps : k) * kDBlockK;
                        const int nmma = (min(kDBlockK, q.K - kk) + 15) / 16;      // what lies past K is filled with zeros
                        const uint64_t a_desc = a_desc0 + static_cast<uint64_t>(s * (kDOperandBytes >> 4));
                        const uint64_t b_desc = b_desc0 + static_cast<uint64_t>(s * (kDOperandBytes >> 4));
#pragma unroll
                        for (int j = 0; j < kDBlockK / 16; ++j)
                            if (j < nmma)
                                tcgen05_mma_f16_pair(tmem + b * kDTile, a_desc + step_a * j, b_desc + kStepB * j, idesc, k > first || j > 0);
                        tcgen05_commit_pair(&sm.empty[s], 3);
                        if (++s == kDStages) {
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
        }
    } else {
        // ------------------------------------------------------------ epilogue warps
        setmaxnreg_inc<216>();
        const int quad = warp & 3;                     // TMEM lane quadrant of this warp
        const int half = warp >> 2;                    // which 128 columns
        const uint64_t streaming = l2_policy_evict_first();      // outputs should not displace operands
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        const uint32_t tmem_empty_leader = map_to_cta(smem_u32(&sm.tmem_empty[0]), 0);
        // boxes of 32 rows x 128 bytes, staged in the 128-byte swizzle for a TMA store that clips at the matrix edges; the
        // boxes' buffers take turns
        int box = 0;
        auto stage_wait = [&]() {
            if (lane == 0) bulk_wait_group_read<kBoxes - 1>();
            __syncwarp();
        };
        auto stage_put = [&](int i, const uint4& v) {
            smem_store(&sm.out_stage[warp][box][0] + lane * 128 + ((i ^ (lane & 7)) * 16), v, sm.out_stage[warp], kBoxes * kDStageBytes);
        };
        auto stage_store = [&](const CUtensorMap* map, int col, int row, bool add = false) {
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
                if (add) tma_add_2d(map, sm.out_stage[warp][box], col, row);
                else tma_store_2d_hint(map, sm.out_stage[warp][box], col, row, streaming);
                bulk_commit_group();
            }
            if (++box == kBoxes) box = 0;
        };
        float common = 1.0f;
        if constexpr (EPI == kDenseScaled || EPI == kDenseLogitGrad) common = dense_common(p.x, sm.common, warp, lane);
        const float2 alpha = pair(p.x.scale * common);           // kDenseScaled: of all sums
        int b = 0;
        uint32_t parity = 0;
        for (int j = 0;; ++j) {
            const DenseWork w = dense_work<kStore>(p, cluster_id, n_clusters, j);
            if (w.q < 0) break;
            const DenseShape& q = p.q[w.q];
            const DenseMaps& m = maps.q[w.q];
            const int tn = w.tn;
            const int in_tile = static_cast<int>(rank) * kDHalf + quad * 32;
            const int row0 = w.row + in_tile;
            const int row = row0 + lane;
            if (!mbar_wait(&sm.tmem_full[b], parity, &sm.abort_flag)) break;       // given up: nothing more is stored
            tcgen05_fence_after();
            auto hand_back = [&]() {
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(tmem_empty_leader + b * 8);
            };
            uint32_t r[32];
            auto read = [&](int col) {
                tmem_ld_32x32b_x32(lanes + b * kDTile + col, r);
                tmem_ld_wait_for(r);
            };
            if constexpr (EPI == kDensePartials) {
                const int col0 = (tn * 2 + half) * q.width, col1 = min(q.N, col0 + q.width);
                const bool any = row0 < q.M && col0 < col1;                    // warp-uniform
                bool alive = true;
                float z[4][32];
                for (int k = w.k0;;) {
                    if (any) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            if (col0 + c * 32 >= col1) break;
                            read(half * q.width + c * 32);
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                z[c][i] = k == w.k0 ? __uint_as_float(r[i]) : z[c][i] + __uint_as_float(r[i]);
                        }
                    }
                    hand_back();
                    k += kDChain;
                    if (k >= w.k1) break;
                    parity ^= b;
                    b ^= 1;
                    alive = mbar_wait(&sm.tmem_full[b], parity, &sm.abort_flag);
                    if (!alive) break;
                    tcgen05_fence_after();
                }
                if (!alive) break;                     // given up: nothing more is stored
                if (any) {
                    const bool row_ok = row < q.M;
                    const int64_t target = row_ok && p.x.targets ? p.x.targets[row] : -1;
                    const int at = target >= p.x.col_base + col0 && target < p.x.col_base + col1
                                       ? static_cast<int>(target - p.x.col_base - col0) : -1;
                    const bool any_here = __any_sync(0xffffffffu, at >= 0);
                    float top = -INFINITY, sum = 0.0f, picked = 0.0f;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            z[c][i] = col0 + c * 32 + i < col1 ? z[c][i] * p.x.scale : -INFINITY;
                            top = fmaxf(top, z[c][i]);
                        }
                        if (any_here) {
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (c * 32 + i == at) picked = z[c][i];
                        }
                    }
                    // a row of nothing but -infinity has sum 0; a NaN passes the maximum by and enters the sum
                    const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        float part = 0.0f;             // four sums of 32
#pragma unroll
                        for (int i = 0; i < 32; ++i) part += dense_exp(z[c][i] - ref);
                        sum += part;
                    }
                    if (row_ok) {
                        p.x.parts[static_cast<int64_t>(tn * 2 + half) * p.x.ld_parts + row] = make_float2(top, sum);
                        if (at >= 0) p.x.picked[row] = picked;
                    }
                }
            } else if (row0 >= q.M || w.k0 == w.k1) {         // warp-uniform: no rows here, or a piece without products
                hand_back();
            } else if constexpr (kStore) {
                const int col0 = tn * kDTile + half * kDHalf;
                const CUtensorMap* out = &m.out[w.seg];
                const int out_row = w.out_row + in_tile;
                const bool k32 = q.out != kDenseBf16;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int col = col0 + c * 32;
                    if (col < q.N) {
                        read(half * kDHalf + c * 32);
                        if constexpr (EPI == kDenseScaled) {
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                const float2 v = __fmul2_rn(make_float2(__uint_as_float(r[i]), __uint_as_float(r[i + 1])), alpha);
                                r[i] = __float_as_uint(v.x);
                                r[i + 1] = __float_as_uint(v.y);
                            }
                        }
                        if (k32 || (c & 1) == 0) stage_wait();
                        if (k32) {
#pragma unroll
                            for (int i = 0; i < 8; ++i) stage_put(i, make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]));
                        } else {
#pragma unroll
                            for (int i = 0; i < 4; ++i) stage_put((c & 1) * 4 + i, dense_pack8(r + 8 * i));
                        }
                    }
                    if (k32 ? col < q.N : (c & 1) != 0 && col - 32 < q.N)
                        stage_store(out, k32 ? col : col - 32, out_row, q.out == kDenseAddF32);
                }
                hand_back();
            } else if constexpr (EPI == kDenseGated) {
                const int col0 = tn * q.width + half * 64, col1 = min(q.N, (tn + 1) * q.width);
                if (col0 < col1) {
                    // a box that the tile's end cuts is written by the threads themselves, eight features at a time
                    const bool keep = p.x.keep != 0, cut = col0 + 64 > col1;
                    uint4 h[8], g8[8], u8[8];
                    auto write = [&](int which, int i, const uint4& v) {
                        if (row < q.M && col0 + i * 8 < col1)
                            *reinterpret_cast<uint4*>(p.x.out[which] + row * p.x.ld_out[which] + col0 + i * 8) = v;
                    };
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t u[32];
                        tmem_ld_32x32b_x32(lanes + b * kDTile + q.width + half * 64 + c * 32, u);
                        read(half * 64 + c * 32);
                        tmem_ld_wait_for(u);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            g8[c * 4 + i] = dense_pack8(r + 8 * i);
                            u8[c * 4 + i] = dense_pack8(u + 8 * i);
                        }
                        with_act(p.x.act, [&](auto act) {
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                r[i] = __float_as_uint(act_value<decltype(act)::value>(__uint_as_float(r[i])) *
                                                       __uint_as_float(u[i]));
                        });
#pragma unroll
                        for (int i = 0; i < 4; ++i) h[c * 4 + i] = dense_pack8(r + 8 * i);
                    }
                    hand_back();
                    auto leave = [&](int which, const uint4 (&v)[8]) {
                        if (cut) {
#pragma unroll
                            for (int i = 0; i < 8; ++i) write(which, i, v[i]);
                        } else {
                            stage_wait();
#pragma unroll
                            for (int i = 0; i < 8; ++i) stage_put(i, v[i]);
                            stage_store(&m.out[which], col0, row0);
                        }
                    };
                    leave(0, h);
                    if (keep) {
                        leave(1, g8);
                        leave(2, u8);
                    }
                } else {
                    hand_back();
                }
            } else {
                // gradients of rows of logits
                const int col0 = (tn * 2 + half) * q.width, col1 = min(q.N, col0 + q.width);
                const bool row_ok = row < q.M;
                const int64_t target = row_ok && p.x.targets ? p.x.targets[row] : -1;
                const int at = target >= p.x.col_base + col0 && target < p.x.col_base + col1
                                   ? static_cast<int>(target - p.x.col_base - col0) : -1;
                const bool any_here = __any_sync(0xffffffffu, at >= 0);
                const float lse = row_ok ? p.x.lse[row] : 0.0f;
                float gl = row_ok && p.x.d_logp && target >= 0 ? p.x.d_logp[row] : 0.0f;
                float gn = row_ok && p.x.d_lse ? p.x.d_lse[row] : 0.0f;
                if (p.x.d_logp && target >= p.x.vocab) gl = NAN;
                const bool zero = (gl == 0.0f && gn == 0.0f);
                gl = __fdiv_rn(gl, common);
                gn = __fdiv_rn(gn, common);
                const float coef = gn - gl;
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    const int col = col0 + c * 32;
                    if (col < p.x.ld_grad) {
                        read(half * kDHalf + c * 32);
                        if ((c & 1) == 0) stage_wait();
                        float z[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            z[i] = coef * dense_exp(__uint_as_float(r[i]) * p.x.scale - lse);
                            if (zero || col + i >= q.N) z[i] = 0.0f;
                        }
                        if (any_here) {
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (c * 32 + i == at) z[i] += gl;
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            stage_put((c & 1) * 4 + i, dense_pack8(reinterpret_cast<uint32_t*>(z) + 8 * i));
                    }
                    if ((c & 1) != 0 && col - 32 < p.x.ld_grad) stage_store(&m.out[0], col - 32, row0);
                }
                hand_back();
            }
            parity ^= b;
            b ^= 1;
        }
        if (lane == 0) bulk_wait_group<0>();
    }

    // neither CTA may leave (or free TMEM) while its peer can still signal it or read its memory
    tcgen05_fence_before();
    __syncthreads();
    cluster_sync_all();
    if (warp == kDMmaWarp) {
        tcgen05_fence_after();
        tmem_dealloc_pair(tmem, 512);
    }
}

}  // namespace mxfp4
