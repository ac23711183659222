// The end of one residual block and the start of the next in one pass over the tokens:
//
//   n = u * rsqrt(mean(u^2) + eps)          (u: the block's output; without w_post: n = u)
//   b = n * w_post,   g = act(gate)         (without a gate: g = 1)
//   y = skip_scale * x + branch_scale * g * b      rounded to the stream's type and stored
//   h = y * rsqrt(mean(y^2) + eps) * w_pre         of the stored y
//
// and its gradient with respect to x, u, the gate and both weights, given dh and dy.  The gradient
// reads the stored y, so it is the gradient of exactly the map the forward pass computed; the two
// root mean squares are formed again from rows that have to be read anyway, so nothing but y is
// kept between the passes.
//
// A row belongs to one CTA (up to 4096 columns, eight per thread) or to a cluster of two or four, which add up
// their sums through distributed shared memory.  Bulk copies keep a ring of rows on their way into shared
// memory while the row at hand goes through its reductions in registers; the vectors every row needs and
// the sums of the weight gradients stay in registers for all of a CTA's rows.  All arithmetic is fp32;
// the outputs are rounded once.
//
// Bound by memory forward (16384 x 4096, bf16 stream, sigmoid gate per element: 117 us for 671 MB, 5.7 TB/s).  Backward the
// registers of the weight gradients leave one CTA of 512 threads per SM, and the one reduction per row stands between its
// loads and stores: 203 to 210 us for 1.07 GB (SiLU gate per element; 5.1 to 5.3 TB/s), a row in 1.8 us; 1003 x 14336 with an
// fp32 stream, where the reduction crosses four CTAs, 73 us for 259 MB (3.6 TB/s), a row in 2.1 us.  Rows that take a
// cluster, 4096 x 14336: forward 125 us for 470 MB (bf16 stream) and 160 for 705 (fp32), backward 256 and 260 for 705
// and 1057 MB.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/mxfp4.h"
#include "host_common.cuh"
#include "ptx_sm100.cuh"
#include "row_io.cuh"
#include "tma_host.cuh"

namespace mxfp4 {

constexpr int kNormMaxWidth = 16384;
constexpr int kNormMaxThreads = 512;
constexpr int kNormMaxCluster = 4;
constexpr int kNormMaxStages = 8;
constexpr int kNormWorkspaceSms = 160;
constexpr int kNormRingBytes = 200 * 1024;       // per SM

struct NormParams {
    const __nv_bfloat16* branch;
    const void* stream;                  // x (forward), y (backward)
    const void* gate;                    // bf16 [tokens x width] or fp32 [width]
    const float* w_post;
    const float* w_pre;
    int64_t ld_branch, ld_stream, ld_gate;
    int32_t tokens;
    int32_t width;
    int32_t cluster;                     // CTAs that share a row
    int32_t cta_chunks;                  // 8-column chunks per CTA
    int32_t gate_act;
    float skip_scale, branch_scale, eps;
    // the ring of rows in shared memory: offsets of the tensors inside a stage, -1 where absent
    int32_t at_stream, at_gate, at_dh, at_dy;
    int32_t stage_bytes, stages;
};

struct NormForwardOut {
    void* y;
    __nv_bfloat16* h;
    int64_t ld_y, ld_h;
};

struct NormBackwardIo {
    const __nv_bfloat16* dh;
    const void* dy;
    void* dx;
    __nv_bfloat16* dbranch;
    void* dgate;                         // bf16 per element; the per-channel gradient goes through `partials`
    float* partials;                     // [cluster][accumulated vector][width]
    int64_t ld_dh, ld_dy, ld_dx, ld_dbranch, ld_dgate;
    int32_t acc_pre, acc_post, acc_gate; // index of the accumulated vector, -1 where none is wanted
    int32_t n_acc;
};

// What a kernel is compiled for: no gate, a gate per channel (its activation is applied once), or a gate per
// element with one of the activations.
enum NormGate { kGateNone, kGateChannel, kGateLinear, kGateSigmoid, kGateSilu };
__host__ __device__ constexpr bool gate_per_element(int gate) { return gate >= kGateLinear; }

// 1 / (1 + e^-x): the reciprocal of infinity is 0, so every finite x and both infinities are fine
__device__ __forceinline__ float sigmoid(float x)
{
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
    return r;
}

template <int GATE>
__device__ __forceinline__ void gate_value_slope(float g, float& v, float& slope)
{
    if (GATE == kGateLinear) {
        v = g;
        slope = 1.0f;
        return;
    }
    const float s = sigmoid(g);
    if (GATE == kGateSigmoid) {
        v = s;
        slope = fmaf(-s, s, s);
    } else {
        v = g * s;
        slope = s * fmaf(g, 1.0f - s, 1.0f);
    }
}

template <int GATE>
__device__ __forceinline__ void gate_pair(const float2& g, float2& v, float2& slope)
{
    gate_value_slope<GATE>(g.x, v.x, slope.x);
    gate_value_slope<GATE>(g.y, v.y, slope.y);
}

// the same with the activation as a value (once per kernel)
__device__ __forceinline__ void gate_pair_of(const float2& g, int act, float2& v, float2& slope)
{
    if (act == MXFP4_GATE_LINEAR) gate_pair<kGateLinear>(g, v, slope);
    else if (act == MXFP4_GATE_SIGMOID) gate_pair<kGateSigmoid>(g, v, slope);
    else gate_pair<kGateSilu>(g, v, slope);
}

constexpr int kNormWarps = kNormMaxThreads / 32;

struct NormShared {
    float red[2][4][kNormMaxCluster * kNormWarps];   // [slot][value][CTA, warp]
    uint64_t sums[2];                    // a slot's values are here: from the CTAs of the cluster, or this CTA's warps
    uint64_t full[kNormMaxStages];
    uint64_t empty[kNormMaxStages];
    int abort_flag;
};

// Where a thread stands: its chunk of eight columns, and the rows its cluster walks.  A thread past the last
// chunk works on the last one with the others and keeps its sums and results to itself.
struct NormPlace {
    int rank;             // of the CTA in its cluster
    int local;            // chunk in the CTA's part of a row
    int col;
    bool active;
    int first, step;      // rows first, first + step, ...
};

template <bool CLUSTER>
__device__ __forceinline__ NormPlace norm_place(const NormParams& p)
{
    NormPlace t;
    t.rank = CLUSTER ? static_cast<int>(cluster_ctarank()) : 0;
    const int here = min(p.cta_chunks, p.width / 8 - t.rank * p.cta_chunks);
    t.active = static_cast<int>(threadIdx.x) < here;
    t.local = t.active ? threadIdx.x : here - 1;
    t.col = (t.rank * p.cta_chunks + t.local) * 8;
    t.first = CLUSTER ? blockIdx.x / p.cluster : blockIdx.x;
    t.step = CLUSTER ? gridDim.x / p.cluster : gridDim.x;
    return t;
}

// Sums over a row of N values (2 or 4) at once, the same in every thread of the cluster.
//
// Inside a warp, exchanges with the lane 16 (and 8) away halve the number of values a lane holds, further
// exchanges finish the one it is left with: value lane / (32 / N), the same in all lanes of that group.
// Every warp leaves its sums in the shared memory of all CTAs of the cluster; then every warp adds all of
// them.  Inside one CTA the forward pass waits for that at an mbarrier and the backward pass at the block's barrier, as
// measured (16384 x 4096 without a gate, both forms in one run): forward 89 us against 93 at the block's barrier,
// backward 165 against 155.  `call` counts the calls: slots alternate, and a slot is written again only after every warp has
// read it (it takes part in the call in between afterwards).
template <int N, bool CLUSTER>
__device__ __forceinline__ void row_sum(float (&v)[N], NormShared& sh, uint32_t& call, int cluster, int rank)
{
    static_assert(N == 2 || N == 4, "two or four values");
    constexpr int kLanes = 32 / N;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int slot = call & 1, value = lane / kLanes, in_group = lane & (kLanes - 1);
    float t;
    if (N == 2) {
        const bool up = lane & 16;
        t = (up ? v[1] : v[0]) + __shfl_xor_sync(0xffffffffu, up ? v[0] : v[1], 16);
    } else {
        const bool up = lane & 16, right = lane & 8;
        const float a = (up ? v[2] : v[0]) + __shfl_xor_sync(0xffffffffu, up ? v[0] : v[2], 16);
        const float b = (up ? v[3] : v[1]) + __shfl_xor_sync(0xffffffffu, up ? v[1] : v[3], 16);
        t = (right ? b : a) + __shfl_xor_sync(0xffffffffu, right ? a : b, 8);
    }
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    const int n = CLUSTER ? cluster * warps : warps;
    if (!CLUSTER) {
        if (in_group == 0) smem_put(sh.red[slot][value], warp, t);
        if (N == 4) {
            __syncthreads();
        } else {
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.sums[slot]);
            (void)mbar_wait_fast(&sh.sums[slot], (call >> 1) & 1, &sh.abort_flag);
        }
    } else {
        if (in_group < cluster && smem_within(sh.red[slot][value], rank * warps + warp))     // to CTA `in_group`
            st_async_f32(map_to_cta(smem_u32(&sh.red[slot][value][rank * warps + warp]), in_group), t,
                         map_to_cta(smem_u32(&sh.sums[slot]), in_group));
        if (threadIdx.x == 0) mbar_arrive_expect_tx(&sh.sums[slot], n * N * 4);
        (void)mbar_wait_fast(&sh.sums[slot], (call >> 1) & 1, &sh.abort_flag);
    }
    ++call;
    t = 0.0f;
    if (!CLUSTER) {
        // at most sixteen warps: one or two entries per lane
        if (in_group < n) t = smem_get(sh.red[slot][value], in_group);
        if (N == 4 && in_group + kLanes < n) t += smem_get(sh.red[slot][value], in_group + kLanes);
    } else {
        for (int j = in_group; j < n; j += kLanes) t += smem_get(sh.red[slot][value], j);
    }
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __shfl_sync(0xffffffffu, t, kLanes * i);
}

template <bool CLUSTER>
__device__ __forceinline__ void norm_setup(NormShared& sh, const NormParams& p)
{
    if (threadIdx.x == 0) {
        sh.abort_flag = 0;
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(&sh.full[s], 1);
            mbar_init(&sh.empty[s], blockDim.x >> 5);
        }
        for (int s = 0; s < 2; ++s) mbar_init(&sh.sums[s], CLUSTER ? 1 : blockDim.x >> 5);
        fence_barrier_init();
    }
    if (CLUSTER) cluster_sync_all();
    else __syncthreads();
    griddep_launch_dependents();
    griddep_wait();
}

// Eight values of a tensor's part of a stage.
__device__ __forceinline__ void stage8(const uint8_t* at, const uint8_t* stage, int bytes, float2 (&v)[4], __nv_bfloat16)
{
    unpack8(smem_load<uint4>(at, stage, bytes), v);
}
__device__ __forceinline__ void stage8(const uint8_t* at, const uint8_t* stage, int bytes, float2 (&v)[4], float)
{
    const float4 a = smem_load<float4>(at, stage, bytes), b = smem_load<float4>(at + 16, stage, bytes);
    v[0] = make_float2(a.x, a.y);
    v[1] = make_float2(a.z, a.w);
    v[2] = make_float2(b.x, b.y);
    v[3] = make_float2(b.z, b.w);
}

// Starts the loads of one row's columns of this CTA into a stage (one thread): whole row pieces as bulk copies.
template <class Stream, int GATE>
__device__ __forceinline__ void norm_issue(const NormParams& p, const NormPlace& t, int row, uint8_t* stage, uint64_t* bar,
                                           const NormBackwardIo* io)
{
    const int col = t.rank * p.cta_chunks * 8;
    const uint32_t n = static_cast<uint32_t>(min(p.cta_chunks * 8, p.width - col));
    const uint32_t half = n * 2, full = n * sizeof(Stream);
    const int64_t r = row;
    uint32_t bytes = half;
    if (p.at_stream >= 0) bytes += full;
    if (gate_per_element(GATE)) bytes += half;
    if (io && p.at_dh >= 0) bytes += half;
    if (io && p.at_dy >= 0) bytes += full;
    mbar_arrive_expect_tx(bar, bytes);
    bulk_load_1d(stage, p.branch + r * p.ld_branch + col, half, bar);
    if (p.at_stream >= 0)
        bulk_load_1d(stage + p.at_stream, static_cast<const Stream*>(p.stream) + r * p.ld_stream + col, full, bar);
    if (gate_per_element(GATE))
        bulk_load_1d(stage + p.at_gate, static_cast<const __nv_bfloat16*>(p.gate) + r * p.ld_gate + col, half, bar);
    if (io && p.at_dh >= 0) bulk_load_1d(stage + p.at_dh, io->dh + r * io->ld_dh + col, half, bar);
    if (io && p.at_dy >= 0)
        bulk_load_1d(stage + p.at_dy, static_cast<const Stream*>(io->dy) + r * io->ld_dy + col, full, bar);
}

// This warp has its part of a stage in registers.
__device__ __forceinline__ void norm_release(NormShared& sh, int s)
{
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(&sh.empty[s]);
}

// Once all warps have: the row that takes the stage next (one thread).
template <class Stream, int GATE>
__device__ __forceinline__ void norm_refill(const NormParams& p, const NormPlace& t, int row, uint8_t* stage, NormShared& sh,
                                            int s, uint32_t parity, const NormBackwardIo* io)
{
    if (threadIdx.x == 0 && row + static_cast<int64_t>(p.stages) * t.step < p.tokens &&
        mbar_wait_fast(&sh.empty[s], parity, &sh.abort_flag))
        norm_issue<Stream, GATE>(p, t, row + p.stages * t.step, stage, &sh.full[s], io);
}

// Walks a [tokens x width] matrix with the rows of a cluster.
template <class T>
struct RowWalk {
    T* at;
    int64_t step;
    __device__ __forceinline__ RowWalk(void* base, int64_t ld, const NormPlace& t)
        : at(static_cast<T*>(base) + t.first * ld + t.col), step(t.step * ld) {}
    __device__ __forceinline__ void next() { at += step; }
};

// Position in the ring.
struct RingPlace {
    int s = 0;
    uint32_t parity = 0;
    __device__ __forceinline__ void next(int stages)
    {
        if (++s == stages) {
            s = 0;
            parity ^= 1u;
        }
    }
};

template <class Stream, int GATE, bool CLUSTER>
__global__ void __launch_bounds__(kNormMaxThreads, 2)
residual_norm_forward_kernel(const __grid_constant__ NormParams p, const __grid_constant__ NormForwardOut out)
{
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ NormShared sh;
    norm_setup<CLUSTER>(sh, p);
    const NormPlace t = norm_place<CLUSTER>(p);
    const float inv_width = 1.0f / static_cast<float>(p.width);
    const bool post = p.w_post != nullptr, pre = p.w_pre != nullptr;
    if (threadIdx.x == 0)
        for (int s = 0; s < p.stages && t.first + s * t.step < p.tokens; ++s)
            norm_issue<Stream, GATE>(p, t, t.first + s * t.step, ring + s * p.stage_bytes, &sh.full[s], nullptr);
    // vectors every row needs
    float2 wb[4], wh[4], w[4];                // branch_scale * w_post * channel gate, w_pre
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        wb[i] = pair(p.branch_scale);
        wh[i] = pair(1.0f);
    }
    if (post) {
        load8(p.w_post + t.col, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) wb[i] = __fmul2_rn(wb[i], w[i]);
    }
    if (GATE == kGateChannel) {
        load8(static_cast<const float*>(p.gate) + t.col, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float2 v, slope;
            gate_pair_of(w[i], p.gate_act, v, slope);
            wb[i] = __fmul2_rn(wb[i], v);
        }
    }
    if (pre) load8(p.w_pre + t.col, wh);
    RowWalk<Stream> y(out.y, out.ld_y, t);
    RowWalk<__nv_bfloat16> h(out.h, out.ld_h, t);
    RingPlace at, ahead;                       // of the row at hand, of the one after it
    uint32_t call = 0;
    // One reduction per row: the sum the first norm of the NEXT row needs, and the one the second norm of this
    // row needs.  The next row's part is read from its stage twice for that, which costs less than a second
    // barrier in every row.
    float sums[2];
    auto look_ahead = [&](int row) {
        sums[0] = 0.0f;
        if (post && row < p.tokens) {
            const uint8_t* stage = ring + ahead.s * p.stage_bytes;
            (void)mbar_wait_fast(&sh.full[ahead.s], ahead.parity, &sh.abort_flag);   // given up: the status word says so
            float2 u[4];
            stage8(stage + t.local * 16, stage, p.stage_bytes, u, __nv_bfloat16());
            float2 sq = __fmul2_rn(u[0], u[0]);
#pragma unroll
            for (int i = 1; i < 4; ++i) sq = __ffma2_rn(u[i], u[i], sq);
            sums[0] = t.active ? sq.x + sq.y : 0.0f;
        }
        ahead.next(p.stages);
    };
    look_ahead(t.first);
    sums[1] = 0.0f;
    if (post) row_sum<2, CLUSTER>(sums, sh, call, p.cluster, t.rank);
    for (int row = t.first; row < p.tokens; row += t.step) {
        const float r_u = post ? rsqrtf(sums[0] * inv_width + p.eps) : 1.0f;
        look_ahead(row + t.step);
        uint8_t* stage = ring + at.s * p.stage_bytes;
        (void)mbar_wait_fast(&sh.full[at.s], at.parity, &sh.abort_flag);
        float2 u[4], x[4], g[4];
        stage8(stage + t.local * 16, stage, p.stage_bytes, u, __nv_bfloat16());
        if (p.at_stream >= 0) {
            stage8(stage + p.at_stream + t.local * (8 * sizeof(Stream)), stage, p.stage_bytes, x, Stream());
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = pair(0.0f);
        }
        if (gate_per_element(GATE)) stage8(stage + p.at_gate + t.local * 16, stage, p.stage_bytes, g, __nv_bfloat16());
        norm_release(sh, at.s);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float2 b = __fmul2_rn(__fmul2_rn(u[i], pair(r_u)), wb[i]);
            if (gate_per_element(GATE)) {
                float2 v, slope;
                gate_pair<GATE>(g[i], v, slope);
                b = __fmul2_rn(b, v);
            }
            u[i] = __ffma2_rn(pair(p.skip_scale), x[i], b);
        }
        store8_round(y.at, u, t.active);
        y.next();
        if (pre) {
            float2 sq = __fmul2_rn(u[0], u[0]);
#pragma unroll
            for (int i = 1; i < 4; ++i) sq = __ffma2_rn(u[i], u[i], sq);
            sums[1] = t.active ? sq.x + sq.y : 0.0f;
        }
        if (post || pre) row_sum<2, CLUSTER>(sums, sh, call, p.cluster, t.rank);
        norm_refill<Stream, GATE>(p, t, row, stage, sh, at.s, at.parity, nullptr);
        if (pre) {
            const float r = rsqrtf(sums[1] * inv_width + p.eps);
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = __fmul2_rn(__fmul2_rn(u[i], pair(r)), wh[i]);
            if (t.active) store8(h.at, u);
            h.next();
        }
        at.next(p.stages);
    }
    if (*static_cast<volatile int*>(&sh.abort_flag)) linger();
    if (CLUSTER) cluster_sync_all();             // no CTA leaves while a peer may still write to its shared memory
}

// Weight gradients: a column belongs to one thread of a cluster, which adds its rows' terms in registers; each
// cluster leaves its sums in the workspace and `sum_partials_kernel` adds them in a fixed order, so the
// result does not depend on scheduling.
template <class Stream, int GATE, bool CLUSTER>
__global__ void __launch_bounds__(kNormMaxThreads, 1)
residual_norm_backward_kernel(const __grid_constant__ NormParams p, const __grid_constant__ NormBackwardIo io)
{
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ NormShared sh;
    norm_setup<CLUSTER>(sh, p);
    const NormPlace t = norm_place<CLUSTER>(p);
    const float inv_width = 1.0f / static_cast<float>(p.width);
    const bool post = p.w_post != nullptr, pre = p.w_pre != nullptr;
    if (threadIdx.x == 0)
        for (int s = 0; s < p.stages && t.first + s * t.step < p.tokens; ++s)
            norm_issue<Stream, GATE>(p, t, t.first + s * t.step, ring + s * p.stage_bytes, &sh.full[s], &io);
    // vectors every row needs, and the sums of the gradients of such vectors
    float2 w_post[4], w_pre[4], gv[4], gs[4];
    float2 acc_post[4], acc_pre[4], acc_gate[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w_post[i] = w_pre[i] = gv[i] = gs[i] = pair(1.0f);
        acc_post[i] = acc_pre[i] = acc_gate[i] = pair(0.0f);
    }
    if (post) load8(p.w_post + t.col, w_post);
    if (pre) load8(p.w_pre + t.col, w_pre);
    if (GATE == kGateChannel) {
        float2 w[4];
        load8(static_cast<const float*>(p.gate) + t.col, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) gate_pair_of(w[i], p.gate_act, gv[i], gs[i]);
    }
    const bool want_dx = t.active && io.dx, want_dbranch = t.active && io.dbranch, want_dgate = t.active && io.dgate;
    RowWalk<Stream> dx(io.dx, io.ld_dx, t);
    RowWalk<__nv_bfloat16> dbranch(io.dbranch, io.ld_dbranch, t), dgate(io.dgate, io.ld_dgate, t);
    RingPlace at, ahead;
    uint32_t call = 0;
    // One reduction per row, as in the forward kernel: sum u^2, sum y^2, sum dh w_pre y of the NEXT row, and the
    // sum of this row's branch gradient times n.
    float m[4];
    auto look_ahead = [&](int row) {
        m[0] = m[1] = m[2] = 0.0f;
        if ((post || pre) && row < p.tokens) {
            const uint8_t* stage = ring + ahead.s * p.stage_bytes;
            (void)mbar_wait_fast(&sh.full[ahead.s], ahead.parity, &sh.abort_flag);   // given up: the status word says so
            float2 u[4], y[4], q[4];
            stage8(stage + t.local * 16, stage, p.stage_bytes, u, __nv_bfloat16());
            float2 uu = __fmul2_rn(u[0], u[0]);
#pragma unroll
            for (int i = 1; i < 4; ++i) uu = __ffma2_rn(u[i], u[i], uu);
            if (t.active) m[0] = uu.x + uu.y;
            if (pre) {
                stage8(stage + p.at_stream + t.local * (8 * sizeof(Stream)), stage, p.stage_bytes, y, Stream());
                stage8(stage + p.at_dh + t.local * 16, stage, p.stage_bytes, q, __nv_bfloat16());
                float2 yy = pair(0.0f), qy = pair(0.0f);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    yy = __ffma2_rn(y[i], y[i], yy);
                    qy = __ffma2_rn(__fmul2_rn(q[i], w_pre[i]), y[i], qy);
                }
                if (t.active) {
                    m[1] = yy.x + yy.y;
                    m[2] = qy.x + qy.y;
                }
            }
        }
        ahead.next(p.stages);
    };
    look_ahead(t.first);
    m[3] = 0.0f;
    if (post || pre) row_sum<4, CLUSTER>(m, sh, call, p.cluster, t.rank);
    for (int row = t.first; row < p.tokens; row += t.step) {
        // a norm that is left out has r = 1, mean = 0 and weights of 1, which leave every value as it is
        const float r_u = post ? rsqrtf(m[0] * inv_width + p.eps) : 1.0f;
        const float r_y = pre ? rsqrtf(m[1] * inv_width + p.eps) : 0.0f;
        const float mean_y = r_y * m[2] * inv_width;               // mean of dh w_pre y / rms(y)
        look_ahead(row + t.step);
        uint8_t* stage = ring + at.s * p.stage_bytes;
        (void)mbar_wait_fast(&sh.full[at.s], at.parity, &sh.abort_flag);
        float2 d[4], u[4], g[4], o[4];
        stage8(stage + t.local * 16, stage, p.stage_bytes, u, __nv_bfloat16());
        if (p.at_dy >= 0) {
            stage8(stage + p.at_dy + t.local * (8 * sizeof(Stream)), stage, p.stage_bytes, d, Stream());
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) d[i] = pair(0.0f);
        }
        if (gate_per_element(GATE)) stage8(stage + p.at_gate + t.local * 16, stage, p.stage_bytes, g, __nv_bfloat16());
        if (pre) {
            float2 y[4], q[4];
            stage8(stage + p.at_stream + t.local * (8 * sizeof(Stream)), stage, p.stage_bytes, y, Stream());
            stage8(stage + p.at_dh + t.local * 16, stage, p.stage_bytes, q, __nv_bfloat16());
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 yh = __fmul2_rn(y[i], pair(r_y));
                acc_pre[i] = __ffma2_rn(q[i], yh, acc_pre[i]);
                d[i] = __ffma2_rn(pair(r_y), __ffma2_rn(yh, pair(-mean_y), __fmul2_rn(q[i], w_pre[i])), d[i]);
            }
        }
        norm_release(sh, at.s);
        if (want_dx) {
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = __fmul2_rn(pair(p.skip_scale), d[i]);
            store8(dx.at, o);
        }
        float2 un = pair(0.0f);                    // sum of the branch gradient's n term
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            d[i] = __fmul2_rn(d[i], pair(p.branch_scale));
            u[i] = __fmul2_rn(u[i], pair(r_u));
            if (GATE != kGateNone) {
                float2 v = gv[i], slope = gs[i];
                if (gate_per_element(GATE)) gate_pair<GATE>(g[i], v, slope);
                o[i] = __fmul2_rn(__fmul2_rn(d[i], u[i]), w_post[i]);
                if (GATE != kGateLinear) o[i] = __fmul2_rn(o[i], slope);
                if (GATE == kGateChannel) acc_gate[i] = __fadd2_rn(acc_gate[i], o[i]);
                d[i] = __fmul2_rn(d[i], v);
            }
            acc_post[i] = __ffma2_rn(d[i], u[i], acc_post[i]);
            d[i] = __fmul2_rn(d[i], w_post[i]);
            un = __ffma2_rn(d[i], u[i], un);
        }
        if (gate_per_element(GATE) && want_dgate) store8(dgate.at, o);
        m[3] = t.active ? un.x + un.y : 0.0f;
        if (post || pre) row_sum<4, CLUSTER>(m, sh, call, p.cluster, t.rank);
        norm_refill<Stream, GATE>(p, t, row, stage, sh, at.s, at.parity, &io);
        if (want_dbranch) {
            const float mean_u = post ? m[3] * inv_width : 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) d[i] = __fmul2_rn(pair(r_u), __ffma2_rn(u[i], pair(-mean_u), d[i]));
            store8(dbranch.at, d);
        }
        dx.next();
        dbranch.next();
        dgate.next();
        at.next(p.stages);
    }
    if (t.active) {
        float* part = io.partials + static_cast<int64_t>(t.first) * io.n_acc * p.width + t.col;
        if (io.acc_pre >= 0) store8(part + static_cast<int64_t>(io.acc_pre) * p.width, acc_pre);
        if (io.acc_post >= 0) store8(part + static_cast<int64_t>(io.acc_post) * p.width, acc_post);
        if (io.acc_gate >= 0) store8(part + static_cast<int64_t>(io.acc_gate) * p.width, acc_gate);
    }
    if (*static_cast<volatile int*>(&sh.abort_flag)) linger();
    if (CLUSTER) cluster_sync_all();             // no CTA leaves while a peer may still write to its shared memory
}

struct SumPartials {
    const float* partials;               // [parts][n_acc][width]
    float* out[3];
    int32_t parts, n_acc, width;
};

// Sum over the CTAs' partial vectors.  A CTA takes 128 columns (a float4 per lane); its warps take
// the parts in turn, then warp 0 adds the warps' sums: always the same order.
constexpr int kSumWarps = 16;
__global__ void __launch_bounds__(kSumWarps * 32) sum_partials_kernel(const SumPartials p)
{
    __shared__ float4 part[kSumWarps][32];
    griddep_launch_dependents();
    griddep_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t row4 = static_cast<int64_t>(p.n_acc) * p.width / 4;       // float4 per part
    const int64_t at = static_cast<int64_t>(blockIdx.x) * 32 + lane;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (at < row4) {
#pragma unroll 4
        for (int i = warp; i < p.parts; i += kSumWarps) {
            const float4 v = reinterpret_cast<const float4*>(p.partials)[i * row4 + at];
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
    }
    smem_put(part[warp], lane, s);
    __syncthreads();
    if (warp == 0 && at < row4) {
        for (int w = 1; w < kSumWarps; ++w) {
            const float4 v = smem_get(part[w], lane);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        const int64_t col = at * 4;
        const int a = static_cast<int>(col / p.width);
        float* out = a == 0 ? p.out[0] : a == 1 ? p.out[1] : p.out[2];
        *reinterpret_cast<float4*>(out + (col - static_cast<int64_t>(a) * p.width)) = s;
    }
}

// Shape of a launch: up to 4096 columns per CTA (eight per thread), a cluster of CTAs for wider rows, and as
// many CTAs per SM as their registers allow; the ring takes what shared memory that leaves.  Rows of 4096
// split over two CTAs of half the threads (twice as many on an SM) measured slower: 16384 x 4096 backward
// 253 us against 200, forward 146 against 137 -- the exchange between the CTAs costs more than the
// independent barriers gain.
struct NormShape {
    int cluster, cta_chunks, threads, per_sm;
};

static NormShape norm_shape(int width, bool backward)
{
    NormShape n;
    n.cluster = width <= 4096 ? 1 : width <= 8192 ? 2 : 4;
    n.cta_chunks = (width / 8 + n.cluster - 1) / n.cluster;
    n.threads = (n.cta_chunks + 31) / 32 * 32;
    const int threads_per_sm = backward ? 512 : 1024;            // 128 / 64 registers each
    n.per_sm = threads_per_sm / n.threads;
    if (n.per_sm > 8) n.per_sm = 8;
    return n;
}

// Clusters of this size the device holds with one CTA per SM; a larger persistent grid would run its last
// clusters as a second wave (of four CTAs, 33 fit on 148 SMs, not 37).
static int resident_clusters(int cluster, int sm_count)
{
    if (cluster == 1) return sm_count;
    static int count[kMaxDevices][2] = {};
    static PerDeviceOnce once[2];
    const int dev = current_device(), k = cluster == 2 ? 0 : 1;
    if (dev < 0) return 0;
    once[k].run(dev, [&] {
        auto kernel = residual_norm_backward_kernel<__nv_bfloat16, kGateNone, true>;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(static_cast<unsigned>(sm_count / cluster * cluster), 1, 1);
        cfg.blockDim = dim3(kNormMaxThreads, 1, 1);
        cfg.dynamicSmemBytes = kNormRingBytes;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = static_cast<unsigned>(cluster);
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        int n = 0;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kNormRingBytes) != cudaSuccess ||
            cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n <= 0) {
            (void)cudaGetLastError();
            n = sm_count / cluster;
        }
        count[dev][k] = n;
        return MXFP4_OK;
    });
    return count[dev][k];
}

// Clusters of a launch (one row at a time each).
static int norm_clusters(const NormShape& n, int64_t tokens, int resident)
{
    const int64_t most = static_cast<int64_t>(n.per_sm) * resident;
    return static_cast<int>(tokens < most ? tokens : most);
}

// Stage layout and ring depth.
static void norm_ring(NormParams* p, const NormShape& n, int stream_bytes, bool gate, bool dh, bool dy)
{
    const int cols = n.cta_chunks * 8;
    int at = cols * 2;
    auto take = [&](bool present, int bytes) {
        const int here = present ? at : -1;
        if (present) at += bytes;
        return here;
    };
    p->cluster = n.cluster;
    p->cta_chunks = n.cta_chunks;
    p->at_stream = take(p->stream != nullptr, cols * stream_bytes);
    p->at_gate = take(gate, cols * 2);
    p->at_dh = take(dh, cols * 2);
    p->at_dy = take(dy, cols * stream_bytes);
    p->stage_bytes = (at + 127) / 128 * 128;
    const int room = kNormRingBytes / n.per_sm / p->stage_bytes;
    p->stages = room < kNormMaxStages ? room : kNormMaxStages;
}

template <class Kernel, class... Args>
static int launch_norm(PerDeviceOnce& once, Kernel kernel, const NormParams& p, const NormShape& n, int clusters,
                       cudaStream_t st, const Args&... args)
{
    const int rc = ensure_smem_attribute(once, kernel, kNormRingBytes);
    if (rc != MXFP4_OK) return rc;
    return launch_kernel_pdl_cluster(kernel, clusters * n.cluster, n.threads, static_cast<size_t>(p.stages) * p.stage_bytes,
                                     n.cluster, st, p, args...) == cudaSuccess
               ? MXFP4_OK : MXFP4_ERR_CUDA;
}

template <class Stream, int GATE>
static int launch_norm_forward(const NormParams& p, const NormForwardOut& out, const NormShape& n, int clusters,
                               cudaStream_t st)
{
    static PerDeviceOnce once[2];
    return n.cluster > 1 ? launch_norm(once[1], residual_norm_forward_kernel<Stream, GATE, true>, p, n, clusters, st, out)
                         : launch_norm(once[0], residual_norm_forward_kernel<Stream, GATE, false>, p, n, clusters, st, out);
}

template <class Stream, int GATE>
static int launch_norm_backward(const NormParams& p, const NormBackwardIo& io, const NormShape& n, int clusters,
                                cudaStream_t st)
{
    static PerDeviceOnce once[2];
    return n.cluster > 1 ? launch_norm(once[1], residual_norm_backward_kernel<Stream, GATE, true>, p, n, clusters, st, io)
                         : launch_norm(once[0], residual_norm_backward_kernel<Stream, GATE, false>, p, n, clusters, st, io);
}

// Calls f with the NormGate of a (checked) description as a constant.
template <class F>
static int with_gate(const mxfp4_norm_desc* n, F&& f)
{
    if (n->gate_kind == MXFP4_GATE_NONE) return f(std::integral_constant<int, kGateNone>());
    if (n->gate_kind == MXFP4_GATE_CHANNEL) return f(std::integral_constant<int, kGateChannel>());
    if (n->gate_act == MXFP4_GATE_LINEAR) return f(std::integral_constant<int, kGateLinear>());
    if (n->gate_act == MXFP4_GATE_SIGMOID) return f(std::integral_constant<int, kGateSigmoid>());
    return f(std::integral_constant<int, kGateSilu>());
}

// What both directions check of the description; `stream` may be absent (forward: nothing is added;
// backward: it is only read for the second norm).
static int norm_params(const mxfp4_norm_desc* n, NormParams* p)
{
    if (!n || !n->branch) return MXFP4_ERR_NULL;
    if (n->gate_kind < MXFP4_GATE_NONE || n->gate_kind > MXFP4_GATE_ELEMENT) return MXFP4_ERR_ENUM;
    if (n->gate_act < MXFP4_GATE_LINEAR || n->gate_act > MXFP4_GATE_SILU) return MXFP4_ERR_ENUM;
    if (n->stream_dtype != MXFP4_OUT_BF16 && n->stream_dtype != MXFP4_OUT_FP32) return MXFP4_ERR_ENUM;
    if (!(n->eps >= 0.0f)) return MXFP4_ERR_ENUM;
    if ((n->gate_kind != MXFP4_GATE_NONE) != (n->gate != nullptr)) return MXFP4_ERR_NULL;
    if (n->tokens <= 0 || n->width <= 0 || n->tokens > 0x7FFF0000) return MXFP4_ERR_SHAPE;
    if (n->width % 8 != 0 || n->width > kNormMaxWidth) return MXFP4_ERR_SHAPE;
    const bool element = n->gate_kind == MXFP4_GATE_ELEMENT;
    if (n->ld_branch < n->width || (n->stream && n->ld_stream < n->width) || (element && n->ld_gate < n->width))
        return MXFP4_ERR_SHAPE;
    if (!aligned16(n->branch) || !aligned16(n->stream) || !aligned16(n->gate) || !aligned16(n->w_post) ||
        !aligned16(n->w_pre))
        return MXFP4_ERR_ALIGN;
    if (n->ld_branch % 8 != 0 || (n->stream && n->ld_stream % 8 != 0) || (element && n->ld_gate % 8 != 0))
        return MXFP4_ERR_ALIGN;
    p->branch = static_cast<const __nv_bfloat16*>(n->branch);
    p->stream = n->stream;
    p->gate = n->gate;
    p->w_post = n->w_post;
    p->w_pre = n->w_pre;
    p->ld_branch = n->ld_branch;
    p->ld_stream = n->ld_stream;
    p->ld_gate = n->ld_gate;
    p->tokens = static_cast<int32_t>(n->tokens);
    p->width = static_cast<int32_t>(n->width);
    p->gate_act = n->gate_act;
    p->skip_scale = n->skip_scale;
    p->branch_scale = n->branch_scale;
    p->eps = n->eps;
    return MXFP4_OK;
}

// Status word of this translation unit's kernels, cleared when it is set.
int residual_norm_take_status(int* status) { return take_unit_status(status); }

// A [tokens x width] output or gradient: leading dimension and alignment.
static int norm_matrix_ok(const void* t, int64_t ld, int64_t width)
{
    if (!t) return MXFP4_OK;
    if (ld < width) return MXFP4_ERR_SHAPE;
    return aligned16(t) && ld % 8 == 0 ? MXFP4_OK : MXFP4_ERR_ALIGN;
}

}  // namespace mxfp4

using namespace mxfp4;

extern "C" {

int mxfp4_residual_norm_forward(const mxfp4_norm_desc* norm, void* y, int64_t ld_y, void* h, int64_t ld_h, void* stream)
{
    NormParams p;
    int rc = norm_params(norm, &p);
    if (rc != MXFP4_OK) return rc;
    if (!y || (p.w_pre != nullptr) != (h != nullptr)) return MXFP4_ERR_NULL;
    if ((rc = norm_matrix_ok(y, ld_y, p.width)) != MXFP4_OK) return rc;
    if ((rc = norm_matrix_ok(h, ld_h, p.width)) != MXFP4_OK) return rc;
    const DeviceInfo& dev = device_info();
    if ((rc = device_status_code(dev)) != MXFP4_OK) return rc;
    const NormForwardOut out = {y, static_cast<__nv_bfloat16*>(h), ld_y, ld_h};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool bf16 = norm->stream_dtype == MXFP4_OUT_BF16;
    const NormShape n = norm_shape(p.width, false);
    norm_ring(&p, n, bf16 ? 2 : 4, norm->gate_kind == MXFP4_GATE_ELEMENT, false, false);
    const int clusters = norm_clusters(n, p.tokens, resident_clusters(n.cluster, dev.sm_count));
    return with_gate(norm, [&](auto gate) {
        constexpr int kGate = decltype(gate)::value;
        return bf16 ? launch_norm_forward<__nv_bfloat16, kGate>(p, out, n, clusters, st)
                    : launch_norm_forward<float, kGate>(p, out, n, clusters, st);
    });
}

// One partial vector per accumulated gradient and cluster; sized for kNormWorkspaceSms SMs, so that it needs no
// device (a launch never uses more).
size_t mxfp4_residual_norm_workspace_bytes(int64_t tokens, int64_t width)
{
    if (tokens <= 0 || width <= 0 || width % 8 != 0 || width > kNormMaxWidth) return 0;
    const NormShape n = norm_shape(static_cast<int>(width), true);
    const int clusters = norm_clusters(n, tokens, kNormWorkspaceSms / n.cluster);
    return static_cast<size_t>(clusters) * 3 * static_cast<size_t>(width) * 4;
}

int mxfp4_residual_norm_backward(const mxfp4_norm_desc* norm, const void* dh, int64_t ld_dh, const void* dy,
                                 int64_t ld_dy, void* dx, int64_t ld_dx, void* dbranch, int64_t ld_dbranch,
                                 void* dgate, int64_t ld_dgate, float* dw_post, float* dw_pre, void* workspace,
                                 size_t workspace_bytes, void* stream)
{
    NormParams p;
    int rc = norm_params(norm, &p);
    if (rc != MXFP4_OK) return rc;
    const bool channel = norm->gate_kind == MXFP4_GATE_CHANNEL;
    if ((p.w_pre != nullptr) != (dh != nullptr) || (p.w_pre && !p.stream) || (!dh && !dy)) return MXFP4_ERR_NULL;
    if ((dw_post && !p.w_post) || (dw_pre && !p.w_pre) || (dgate && norm->gate_kind == MXFP4_GATE_NONE))
        return MXFP4_ERR_NULL;
    if ((rc = norm_matrix_ok(dh, ld_dh, p.width)) != MXFP4_OK || (rc = norm_matrix_ok(dy, ld_dy, p.width)) != MXFP4_OK ||
        (rc = norm_matrix_ok(dx, ld_dx, p.width)) != MXFP4_OK ||
        (rc = norm_matrix_ok(dbranch, ld_dbranch, p.width)) != MXFP4_OK ||
        (rc = norm_matrix_ok(dgate, channel ? p.width : ld_dgate, p.width)) != MXFP4_OK)
        return rc;
    if (!aligned16(dw_post) || !aligned16(dw_pre) || !aligned16(workspace)) return MXFP4_ERR_ALIGN;

    NormBackwardIo io;
    io.dh = static_cast<const __nv_bfloat16*>(dh);
    io.dy = dy;
    io.dx = dx;
    io.dbranch = static_cast<__nv_bfloat16*>(dbranch);
    io.dgate = dgate;
    io.partials = static_cast<float*>(workspace);
    io.ld_dh = ld_dh;
    io.ld_dy = ld_dy;
    io.ld_dx = ld_dx;
    io.ld_dbranch = ld_dbranch;
    io.ld_dgate = ld_dgate;
    SumPartials sum = {};
    io.n_acc = 0;
    io.acc_pre = io.acc_post = io.acc_gate = -1;
    if (dw_pre) sum.out[io.acc_pre = io.n_acc++] = dw_pre;
    if (dw_post) sum.out[io.acc_post = io.n_acc++] = dw_post;
    if (channel && dgate) sum.out[io.acc_gate = io.n_acc++] = static_cast<float*>(dgate);
    if (io.n_acc > 0 && (!workspace || workspace_bytes < mxfp4_residual_norm_workspace_bytes(p.tokens, p.width)))
        return MXFP4_ERR_WORKSPACE;
    const DeviceInfo& dev = device_info();
    if ((rc = device_status_code(dev)) != MXFP4_OK) return rc;
    const bool bf16 = norm->stream_dtype == MXFP4_OUT_BF16;
    const NormShape n = norm_shape(p.width, true);
    if (!p.w_pre) p.stream = nullptr;            // y is only read for the second norm
    norm_ring(&p, n, bf16 ? 2 : 4, norm->gate_kind == MXFP4_GATE_ELEMENT, dh != nullptr, dy != nullptr);
    const int fit = resident_clusters(n.cluster, dev.sm_count), room = kNormWorkspaceSms / n.cluster;
    const int grid = norm_clusters(n, p.tokens, fit < room ? fit : room);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    rc = with_gate(norm, [&](auto gate) {
        constexpr int kGate = decltype(gate)::value;
        return bf16 ? launch_norm_backward<__nv_bfloat16, kGate>(p, io, n, grid, st)
                    : launch_norm_backward<float, kGate>(p, io, n, grid, st);
    });
    if (rc != MXFP4_OK || io.n_acc == 0) return rc;
    sum.partials = io.partials;
    sum.parts = grid;
    sum.n_acc = io.n_acc;
    sum.width = p.width;
    const int64_t row4 = static_cast<int64_t>(io.n_acc) * p.width / 4;
    return launch_kernel_pdl(sum_partials_kernel, static_cast<int>((row4 + 31) / 32), kSumWarps * 32, 0, st, sum) ==
                   cudaSuccess
               ? MXFP4_OK : MXFP4_ERR_CUDA;
}

}  // extern "C"
