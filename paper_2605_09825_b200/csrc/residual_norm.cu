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
// One CTA walks whole rows: every tensor is read once in 16-byte loads and stays in registers
// between the reductions over the row.  All arithmetic is fp32; the outputs are rounded once.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/mxfp4.h"
#include "host_common.cuh"
#include "ptx_sm100.cuh"
#include "row_io.cuh"
#include "tma_host.cuh"

namespace mxfp4 {

constexpr int kNormMaxWidth = 16384;
constexpr int kNormMaxThreads = 1024;

struct NormParams {
    const __nv_bfloat16* branch;
    const void* stream;                  // x (forward), y (backward)
    const void* gate;                    // bf16 [tokens x width] or fp32 [width]
    const float* w_post;
    const float* w_pre;
    int64_t ld_branch, ld_stream, ld_gate;
    int64_t tokens;
    int32_t width;
    int32_t gate_kind, gate_act;
    float skip_scale, branch_scale, eps;
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
    __nv_bfloat16* dgate;                // per element; the per-channel gradient goes through `partials`
    float* partials;                     // [CTA][accumulated vector][width]
    int64_t ld_dh, ld_dy, ld_dx, ld_dbranch, ld_dgate;
    int32_t acc_pre, acc_post, acc_gate; // index of the accumulated vector, -1 where none is wanted
    int32_t n_acc;
};

// Sum of up to three values over the CTA, the same in every thread.  `slot` alternates with every
// call so that one barrier per reduction is enough: a slot is written again only after the
// barrier of the reduction in between.
template <int N>
__device__ __forceinline__ void block_sum(float (&v)[N], float* red, int& slot)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    float* r = red + slot * (3 * 32);
    if (lane == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) r[i * 32 + warp] = v[i];
    slot ^= 1;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lane < warps ? r[i * 32 + lane] : 0.0f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
}

// 1 / (1 + e^-x): the quotient of 1 and infinity is 0, so every finite x and both infinities are fine
__device__ __forceinline__ float sigmoid(float x) { return __fdividef(1.0f, 1.0f + __expf(-x)); }

__device__ __forceinline__ float gate_value(float g, int act)
{
    if (act == MXFP4_GATE_LINEAR) return g;
    const float s = sigmoid(g);
    return act == MXFP4_GATE_SIGMOID ? s : g * s;
}

__device__ __forceinline__ void gate_value_slope(float g, int act, float& v, float& slope)
{
    if (act == MXFP4_GATE_LINEAR) {
        v = g;
        slope = 1.0f;
        return;
    }
    const float s = sigmoid(g);
    if (act == MXFP4_GATE_SIGMOID) {
        v = s;
        slope = s * (1.0f - s);
    } else {
        v = g * s;
        slope = s * (1.0f + g * (1.0f - s));
    }
}

// Gate of the eight columns of one chunk (1 without a gate).
__device__ __forceinline__ void load_gate(const NormParams& p, int64_t row, int col, float (&g)[8])
{
    if (p.gate_kind == MXFP4_GATE_ELEMENT) {
        load8(static_cast<const __nv_bfloat16*>(p.gate) + row * p.ld_gate + col, g);
    } else if (p.gate_kind == MXFP4_GATE_CHANNEL) {
        load8_cached(static_cast<const float*>(p.gate) + col, g);
    }
}

template <class Stream, int C>
__global__ void __launch_bounds__(C == 1 ? kNormMaxThreads / 2 : kNormMaxThreads, 1)
residual_norm_forward_kernel(const NormParams p, const NormForwardOut out)
{
    __shared__ float red[2 * 3 * 32];
    griddep_launch_dependents();
    griddep_wait();
    const int chunks = p.width >> 3;
    const float inv_width = 1.0f / static_cast<float>(p.width);
    int slot = 0;
    for (int64_t row = blockIdx.x; row < p.tokens; row += gridDim.x) {
        float u[C][8], x[C][8], g[C][8];
        float ss[1] = {0.0f};
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int chunk = threadIdx.x + c * blockDim.x;
            if (chunk < chunks) {
                load8(p.branch + row * p.ld_branch + chunk * 8, u[c]);
                if (p.stream) load8(static_cast<const Stream*>(p.stream) + row * p.ld_stream + chunk * 8, x[c]);
                load_gate(p, row, chunk * 8, g[c]);
#pragma unroll
                for (int i = 0; i < 8; ++i) ss[0] += u[c][i] * u[c][i];
            }
        }
        float r = 1.0f;
        if (p.w_post) {
            block_sum(ss, red, slot);
            r = rsqrtf(ss[0] * inv_width + p.eps);
        }
        ss[0] = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int chunk = threadIdx.x + c * blockDim.x;
            if (chunk < chunks) {
                float w[8];
                if (p.w_post) load8_cached(p.w_post + chunk * 8, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float b = u[c][i];
                    if (p.w_post) b = b * r * w[i];
                    if (p.gate_kind != MXFP4_GATE_NONE) b *= gate_value(g[c][i], p.gate_act);
                    b *= p.branch_scale;
                    if (p.stream) b = fmaf(p.skip_scale, x[c][i], b);
                    u[c][i] = b;
                }
                store8(static_cast<Stream*>(out.y) + row * out.ld_y + chunk * 8, u[c]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    u[c][i] = as_stored<Stream>(u[c][i]);
                    ss[0] += u[c][i] * u[c][i];
                }
            }
        }
        if (p.w_pre) {
            block_sum(ss, red, slot);
            r = rsqrtf(ss[0] * inv_width + p.eps);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int chunk = threadIdx.x + c * blockDim.x;
                if (chunk < chunks) {
                    float w[8];
                    load8_cached(p.w_pre + chunk * 8, w);
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] *= u[c][i] * r;
                    store8(out.h + row * out.ld_h + chunk * 8, w);
                }
            }
        }
    }
}

// Weight gradients: a column belongs to one thread, which adds its rows' terms to fp32 sums in
// shared memory; each CTA leaves its sums in the workspace and `sum_partials_kernel` adds them in a
// fixed order, so the result does not depend on scheduling.  (Two float4 planes per vector: with
// the eight values of a chunk side by side every second bank would be hit twice.)
__device__ __forceinline__ void accumulate8(float* acc, int chunks, int chunk, const float (&v)[8])
{
    float4* lo = reinterpret_cast<float4*>(acc) + chunk;
    float4* hi = lo + chunks;
    float4 a = *lo, b = *hi;
    a.x += v[0]; a.y += v[1]; a.z += v[2]; a.w += v[3];
    b.x += v[4]; b.y += v[5]; b.z += v[6]; b.w += v[7];
    *lo = a;
    *hi = b;
}

template <class Stream, int C>
__global__ void __launch_bounds__(C == 1 ? kNormMaxThreads / 2 : kNormMaxThreads, 1)
residual_norm_backward_kernel(const NormParams p, const NormBackwardIo io)
{
    extern __shared__ __align__(16) float acc_all[];       // [accumulated vector][width]
    __shared__ float red[2 * 3 * 32];
    griddep_launch_dependents();
    griddep_wait();
    const int chunks = p.width >> 3;
    const float inv_width = 1.0f / static_cast<float>(p.width);
    int slot = 0;
    float* acc_pre = acc_all + static_cast<int64_t>(io.acc_pre) * p.width;
    float* acc_post = acc_all + static_cast<int64_t>(io.acc_post) * p.width;
    float* acc_gate = acc_all + static_cast<int64_t>(io.acc_gate) * p.width;
    for (int i = threadIdx.x; i < io.n_acc * p.width; i += blockDim.x) acc_all[i] = 0.0f;
    __syncthreads();

    for (int64_t row = blockIdx.x; row < p.tokens; row += gridDim.x) {
        float d[C][8], u[C][8], y[C][8], q[C][8];
        float s[3] = {0.0f, 0.0f, 0.0f};           // sum u^2, sum y^2, sum dh w_pre y
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int chunk = threadIdx.x + c * blockDim.x;
            if (chunk < chunks) {
                const int64_t col = chunk * 8;
                load8(p.branch + row * p.ld_branch + col, u[c]);
#pragma unroll
                for (int i = 0; i < 8; ++i) s[0] += u[c][i] * u[c][i];
                if (p.w_pre) {
                    load8(static_cast<const Stream*>(p.stream) + row * p.ld_stream + col, y[c]);
                    load8(io.dh + row * io.ld_dh + col, q[c]);
                    float w[8];
                    load8_cached(p.w_pre + col, w);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        s[1] += y[c][i] * y[c][i];
                        s[2] += q[c][i] * w[i] * y[c][i];
                    }
                }
                if (io.dy) {
                    load8(static_cast<const Stream*>(io.dy) + row * io.ld_dy + col, d[c]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[c][i] = 0.0f;
                }
            }
        }
        float r_u = 1.0f, r_y = 0.0f, mean_y = 0.0f;
        if (p.w_post || p.w_pre) {
            block_sum(s, red, slot);
            if (p.w_post) r_u = rsqrtf(s[0] * inv_width + p.eps);
            if (p.w_pre) {
                r_y = rsqrtf(s[1] * inv_width + p.eps);
                mean_y = r_y * s[2] * inv_width;                   // mean of dh w_pre y / rms(y)
            }
        }
        float t[1] = {0.0f};                       // sum of the branch gradient's n term
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int chunk = threadIdx.x + c * blockDim.x;
            if (chunk < chunks) {
                const int64_t col = chunk * 8;
                if (p.w_pre) {
                    float w[8];
                    load8_cached(p.w_pre + col, w);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float yh = y[c][i] * r_y;
                        d[c][i] += r_y * (q[c][i] * w[i] - yh * mean_y);
                        w[i] = q[c][i] * yh;
                    }
                    if (io.acc_pre >= 0) accumulate8(acc_pre, chunks, chunk, w);
                }
                float o[8];
                if (io.dx) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) o[i] = p.skip_scale * d[c][i];
                    store8(static_cast<Stream*>(io.dx) + row * io.ld_dx + col, o);
                }
                float w[8];
                if (p.w_post) load8_cached(p.w_post + col, w);
                if (p.gate_kind != MXFP4_GATE_NONE) {
                    load_gate(p, row, chunk * 8, o);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float v, slope;
                        gate_value_slope(o[i], p.gate_act, v, slope);
                        const float e = p.branch_scale * d[c][i];
                        float b = u[c][i];
                        if (p.w_post) b *= r_u * w[i];
                        o[i] = e * b * slope;
                        d[c][i] = e * v;
                    }
                    if (io.dgate) store8(io.dgate + row * io.ld_dgate + col, o);
                    if (io.acc_gate >= 0) accumulate8(acc_gate, chunks, chunk, o);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[c][i] *= p.branch_scale;
                }
                if (p.w_post) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        u[c][i] *= r_u;
                        o[i] = d[c][i] * u[c][i];
                        d[c][i] *= w[i];
                        t[0] += d[c][i] * u[c][i];
                    }
                    if (io.acc_post >= 0) accumulate8(acc_post, chunks, chunk, o);
                }
            }
        }
        float mean_u = 0.0f;
        if (p.w_post) {
            block_sum(t, red, slot);
            mean_u = t[0] * inv_width;
        }
        if (io.dbranch) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int chunk = threadIdx.x + c * blockDim.x;
                if (chunk < chunks) {
                    if (p.w_post)
#pragma unroll
                        for (int i = 0; i < 8; ++i) d[c][i] = r_u * (d[c][i] - u[c][i] * mean_u);
                    store8(io.dbranch + row * io.ld_dbranch + chunk * 8, d[c]);
                }
            }
        }
    }
    // a thread wrote and reads only its own columns
    for (int a = 0; a < io.n_acc; ++a) {
        const float4* src = reinterpret_cast<const float4*>(acc_all + static_cast<int64_t>(a) * p.width);
        float4* dst = reinterpret_cast<float4*>(io.partials + (static_cast<int64_t>(blockIdx.x) * io.n_acc + a) * p.width);
        for (int chunk = threadIdx.x; chunk < chunks; chunk += blockDim.x) {
            dst[2 * chunk] = src[chunk];
            dst[2 * chunk + 1] = src[chunks + chunk];
        }
    }
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
    part[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && at < row4) {
        for (int w = 1; w < kSumWarps; ++w) {
            const float4 v = part[w][lane];
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        const int64_t col = at * 4;
        const int a = static_cast<int>(col / p.width);
        *reinterpret_cast<float4*>(p.out[a] + (col - static_cast<int64_t>(a) * p.width)) = s;
    }
}

// Threads per row and 8-column chunks per thread: one chunk each up to 512 threads, two beyond.
static int norm_chunks_per_thread(int width) { return width <= 4096 ? 1 : 2; }

static int norm_threads(int width)
{
    const int c = norm_chunks_per_thread(width);
    const int need = (width / 8 + c - 1) / c;
    return (need + 31) / 32 * 32;
}

static int norm_backward_ctas(int64_t tokens, int width, int n_acc, int sm_count)
{
    // resident CTAs: 64 registers per thread and the shared accumulators
    const int by_threads = 1024 / norm_threads(width);
    const int by_smem = n_acc > 0 ? (200 * 1024) / (n_acc * width * 4 + 2048) : by_threads;
    int per_sm = by_threads < by_smem ? by_threads : by_smem;
    if (per_sm > 4) per_sm = 4;
    if (per_sm < 1) per_sm = 1;
    const int64_t ctas = static_cast<int64_t>(per_sm) * sm_count;
    return static_cast<int>(tokens < ctas ? tokens : ctas);
}

template <class Stream, int C>
static int launch_norm_forward(const NormParams& p, const NormForwardOut& out, int sm_count, cudaStream_t st)
{
    const int64_t most = static_cast<int64_t>(sm_count) * 64;
    const int grid = static_cast<int>(p.tokens < most ? p.tokens : most);
    return launch_kernel_pdl(residual_norm_forward_kernel<Stream, C>, grid, norm_threads(p.width), 0, st, p, out) ==
                   cudaSuccess
               ? MXFP4_OK : MXFP4_ERR_CUDA;
}

template <class Stream, int C>
static int launch_norm_backward(const NormParams& p, const NormBackwardIo& io, int grid, cudaStream_t st)
{
    static PerDeviceOnce once;
    const size_t most = static_cast<size_t>(3) * kNormMaxWidth * 4;
    const int rc = ensure_smem_attribute(once, residual_norm_backward_kernel<Stream, C>, most);
    if (rc != MXFP4_OK) return rc;
    const size_t smem = static_cast<size_t>(io.n_acc) * p.width * 4;
    return launch_kernel_pdl(residual_norm_backward_kernel<Stream, C>, grid, norm_threads(p.width), smem, st, p, io) ==
                   cudaSuccess
               ? MXFP4_OK : MXFP4_ERR_CUDA;
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
    if (n->tokens <= 0 || n->width <= 0 || n->tokens > 0x7FFFFFFF) return MXFP4_ERR_SHAPE;
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
    p->tokens = n->tokens;
    p->width = static_cast<int32_t>(n->width);
    p->gate_kind = n->gate_kind;
    p->gate_act = n->gate_act;
    p->skip_scale = n->skip_scale;
    p->branch_scale = n->branch_scale;
    p->eps = n->eps;
    return MXFP4_OK;
}

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
    const bool one = norm_chunks_per_thread(p.width) == 1;
    if (norm->stream_dtype == MXFP4_OUT_BF16)
        return one ? launch_norm_forward<__nv_bfloat16, 1>(p, out, dev.sm_count, st)
                   : launch_norm_forward<__nv_bfloat16, 2>(p, out, dev.sm_count, st);
    return one ? launch_norm_forward<float, 1>(p, out, dev.sm_count, st)
               : launch_norm_forward<float, 2>(p, out, dev.sm_count, st);
}

// One partial vector per accumulated gradient and CTA; sized for the largest grid any device of
// this kind runs, so that it needs no device.
size_t mxfp4_residual_norm_workspace_bytes(int64_t tokens, int64_t width)
{
    if (tokens <= 0 || width <= 0 || width % 8 != 0 || width > kNormMaxWidth) return 0;
    const int64_t ctas = tokens < 4 * 160 ? tokens : 4 * 160;
    return static_cast<size_t>(ctas) * 3 * static_cast<size_t>(width) * 4;
}

int mxfp4_residual_norm_backward(const mxfp4_norm_desc* norm, const void* dh, int64_t ld_dh, const void* dy,
                                 int64_t ld_dy, void* dx, int64_t ld_dx, void* dbranch, int64_t ld_dbranch,
                                 void* dgate, int64_t ld_dgate, float* dw_post, float* dw_pre, void* workspace,
                                 size_t workspace_bytes, void* stream)
{
    NormParams p;
    int rc = norm_params(norm, &p);
    if (rc != MXFP4_OK) return rc;
    if ((p.w_pre != nullptr) != (dh != nullptr) || (p.w_pre && !p.stream) || (!dh && !dy)) return MXFP4_ERR_NULL;
    if ((dw_post && !p.w_post) || (dw_pre && !p.w_pre) || (dgate && p.gate_kind == MXFP4_GATE_NONE))
        return MXFP4_ERR_NULL;
    const bool channel = p.gate_kind == MXFP4_GATE_CHANNEL;
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
    io.dgate = channel ? nullptr : static_cast<__nv_bfloat16*>(dgate);
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
    const int sms = dev.sm_count < 160 ? dev.sm_count : 160;              // what the workspace is sized for
    const int grid = norm_backward_ctas(p.tokens, p.width, io.n_acc, sms);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool one = norm_chunks_per_thread(p.width) == 1;
    if (norm->stream_dtype == MXFP4_OUT_BF16)
        rc = one ? launch_norm_backward<__nv_bfloat16, 1>(p, io, grid, st)
                 : launch_norm_backward<__nv_bfloat16, 2>(p, io, grid, st);
    else
        rc = one ? launch_norm_backward<float, 1>(p, io, grid, st) : launch_norm_backward<float, 2>(p, io, grid, st);
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
