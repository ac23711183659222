// The global norm of many gradient tensors, and clipping by it (see include/mxfp4.h).
//
// The tensors are cut into blocks of 16384 elements; their descriptors travel as a kernel argument, so a call copies nothing
// to the device and can be captured.  Squares are added in fp32 over the eight or four elements of a 16-byte piece and in
// fp64 beyond that; a piece whose sum leaves fp32's range, or falls where fp32's squares lose bits, is added in fp64
// throughout.  A fixed number of CTAs take blocks in turn and write one partial sum each, and one CTA adds these in
// their order: results do not depend on scheduling.
//
// Bound by memory: 218 million bf16 elements, norm and clipped copy, 212 us for 1.31 GB, of which the second pass over the
// gradients is a third.  Clipping takes a CTA per block, in the device's own order: the blocks being written stay close together
// (130 us; 136 from CTAs that stay and take blocks in turn), the last blocks first.  Keeping what the first pass read last
// in L2 by eviction priorities was worth 1 %.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>

#include "../../include/mxfp4.h"
#include "host_common.cuh"
#include "ptx_sm100.cuh"
#include "row_io.cuh"
#include "tma_host.cuh"

namespace mxfp4 {

constexpr int kNormBlock = 16384;                  // elements
constexpr int kNormThreads = 256;
constexpr int kNormWarps = kNormThreads / 32;
constexpr int kNormUnroll = 8;                     // 16-byte pieces in flight per thread
constexpr int kClipUnroll = 4;
constexpr int kNormCtas = 592;                     // four per SM; a constant, so that results do not depend on the device
constexpr int kNormMostTensors = 640;              // per launch: 30 KB of arguments

struct GradTensor {
    const void* in;
    void* out;
    int64_t numel;
    int32_t in32, out32;         // fp32, otherwise bf16
    int32_t first_block;
};

template <int N>
struct GradNormParams {
    double* parts;               // of this launch: [kNormCtas]
    int32_t count, blocks;
    const float* norm;
    float max_norm, eps;
    GradTensor t[N];
};

// The tensor a block belongs to.
template <int N>
__device__ __forceinline__ int norm_tensor_of(const GradNormParams<N>& p, int block)
{
    int lo = 0, hi = p.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.t[mid].first_block <= block) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ double square64(float v) { return static_cast<double>(v) * static_cast<double>(v); }

// The elements of a 16-byte piece as pairs.
template <class T>
__device__ __forceinline__ void piece_values(const uint4& w, float2 (&v)[8 / sizeof(T)])
{
    if constexpr (sizeof(T) == 2) {
        unpack8(w, v);
    } else {
        v[0] = make_float2(__uint_as_float(w.x), __uint_as_float(w.y));
        v[1] = make_float2(__uint_as_float(w.z), __uint_as_float(w.w));
    }
}

template <class T>
__device__ __forceinline__ float piece_squares(const uint4& w)
{
    constexpr int kPairs = 8 / sizeof(T);
    float2 v[kPairs], s = make_float2(0.0f, 0.0f);
    piece_values<T>(w, v);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) s = __ffma2_rn(v[i], v[i], s);
    return s.x + s.y;
}

template <class T>
__device__ __noinline__ double piece_squares64(uint4 w)
{
    constexpr int kPairs = 8 / sizeof(T);
    float2 v[kPairs];
    piece_values<T>(w, v);
    double s = 0.0;
    for (int i = 0; i < kPairs; ++i) s += square64(v[i].x) + square64(v[i].y);
    return s;
}

template <class T>
__device__ __forceinline__ float as_float(T v)
{
    if constexpr (sizeof(T) == 2) return __bfloat162float(v);
    else return v;
}

// Elements before the first 16-byte boundary.
template <class T>
__device__ __forceinline__ int head_of(const T* p, int n)
{
    return min(n, static_cast<int>(((16u - (reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) / sizeof(T)));
}

template <class T>
__device__ __forceinline__ double block_squares(const T* x, int n)
{
    constexpr int kPer = 16 / sizeof(T);
    double sum = 0.0;
    const int head = head_of(x, n), pieces = (n - head) / kPer, tail = head + pieces * kPer;
    const T* body = x + head;
    for (int i = threadIdx.x; i < pieces; i += kNormThreads * kNormUnroll) {
        uint4 w[kNormUnroll];
#pragma unroll
        for (int u = 0; u < kNormUnroll; ++u)
            w[u] = i + u * kNormThreads < pieces ? ld_stream(body + (i + u * kNormThreads) * kPer) : make_uint4(0u, 0u, 0u, 0u);
        float s[kNormUnroll], least = INFINITY, most = 0.0f;
#pragma unroll
        for (int u = 0; u < kNormUnroll; ++u) {
            s[u] = piece_squares<T>(w[u]);
            least = fminf(least, s[u]);
            most = fmaxf(most, s[u]);
            if (s[u] != s[u]) most = INFINITY;
        }
        if (least > 0x1p-80f && most < INFINITY) {
            double d[kNormUnroll];
#pragma unroll
            for (int u = 0; u < kNormUnroll; ++u) d[u] = static_cast<double>(s[u]);
#pragma unroll
            for (int k = 1; k < kNormUnroll; k *= 2)
#pragma unroll
                for (int u = 0; u + k < kNormUnroll; u += 2 * k) d[u] += d[u + k];
            sum += d[0];
        } else {
            // zeros (the block's end among them), or squares that fp32 does not hold
#pragma unroll
            for (int u = 0; u < kNormUnroll; ++u) {
                constexpr uint32_t kBits = sizeof(T) == 2 ? 0x7FFF7FFFu : 0x7FFFFFFFu;
                if (((w[u].x | w[u].y | w[u].z | w[u].w) & kBits) != 0)
                    sum += s[u] > 0x1p-80f && s[u] < INFINITY ? static_cast<double>(s[u]) : piece_squares64<T>(w[u]);
            }
        }
    }
    if (threadIdx.x < head) sum += square64(as_float(x[threadIdx.x]));
    if (tail + static_cast<int>(threadIdx.x) < n) sum += square64(as_float(x[tail + threadIdx.x]));
    return sum;
}

__device__ __forceinline__ double warp_sum(double v)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

template <int N>
__global__ void __launch_bounds__(kNormThreads, 4) grad_norm_kernel(const __grid_constant__ GradNormParams<N> p)
{
    __shared__ double part[kNormWarps];
    griddep_launch_dependents();
    griddep_wait();
    double sum = 0.0;
    for (int b = blockIdx.x; b < p.blocks; b += kNormCtas) {
        const GradTensor& t = p.t[norm_tensor_of(p, b)];
        const int64_t at = static_cast<int64_t>(b - t.first_block) * kNormBlock;
        const int n = static_cast<int>(min(t.numel - at, static_cast<int64_t>(kNormBlock)));
        sum += t.in32 ? block_squares(static_cast<const float*>(t.in) + at, n)
                      : block_squares(static_cast<const __nv_bfloat16*>(t.in) + at, n);
    }
    sum = warp_sum(sum);
    if ((threadIdx.x & 31) == 0) smem_put(part, threadIdx.x >> 5, sum);
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kNormWarps; ++w) sum += smem_get(part, w);
        p.parts[blockIdx.x] = sum;
    }
}

// The norm from the partial sums of all launches.
__global__ void __launch_bounds__(kNormThreads) grad_norm_join_kernel(const double* parts, int n, float* norm)
{
    __shared__ double part[kNormWarps];
    griddep_launch_dependents();
    griddep_wait();
    double sum = 0.0;
    for (int i = threadIdx.x; i < n; i += kNormThreads) sum += parts[i];
    sum = warp_sum(sum);
    if ((threadIdx.x & 31) == 0) smem_put(part, threadIdx.x >> 5, sum);
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < kNormWarps; ++w) sum += smem_get(part, w);
    *norm = static_cast<float>(sqrt(sum));
}

// What gradients are multiplied by: `factor`, then `step`.  A factor far below the normal numbers (the limit of a norm that
// exploded) would have lost its bits: it is held 2^64 times as large then, and step is 2^-64.
struct ClipFactor {
    float factor, step;
};

__device__ __forceinline__ ClipFactor clip_factor(float norm, float max_norm, float eps)
{
    constexpr float kLargest = 3.402823466e38f;
    ClipFactor f = {1.0f, 1.0f};
    if (!(norm <= kLargest)) return f;                 // not finite: as they are
    const float total = norm + eps, share = max_norm / total;
    if (total <= kLargest && !(share < 0x1p-100f)) {
        if (share < 1.0f) f.factor = share;
        return f;
    }
    const double exact = static_cast<double>(max_norm) / (static_cast<double>(norm) + static_cast<double>(eps));
    if (exact < 0x1p-100) {
        f.factor = static_cast<float>(exact * 0x1p64);
        f.step = 0x1p-64f;
    } else if (exact < 1.0) {
        f.factor = static_cast<float>(exact);
    }
    return f;
}

template <class In, class Out>
__device__ __forceinline__ void block_scale(const In* x, Out* y, int n, const ClipFactor& f)
{
    constexpr int kPer = 16 / (sizeof(In) < sizeof(Out) ? sizeof(In) : sizeof(Out));       // elements per step: 16 or 32 bytes
    const int head = head_of(x, n);
    const bool vectors = kPer == 8 ? (reinterpret_cast<uintptr_t>(y + head) & 15u) == 0 && (reinterpret_cast<uintptr_t>(x + head) & 15u) == 0
                                   : (reinterpret_cast<uintptr_t>(y + head) & 15u) == 0;
    if (!vectors || f.step != 1.0f) {
        for (int i = threadIdx.x; i < n; i += kNormThreads) {
            const float v = as_float(x[i]) * f.factor * f.step;
            if constexpr (sizeof(Out) == 2) y[i] = __float2bfloat16_rn(v);
            else y[i] = v;
        }
        return;
    }
    const int pieces = (n - head) / kPer, tail = head + pieces * kPer;
    for (int i = threadIdx.x; i < pieces; i += kNormThreads * kClipUnroll) {
        uint4 w[kClipUnroll][sizeof(In) * kPer / 16];
#pragma unroll
        for (int u = 0; u < kClipUnroll; ++u) {
            if (i + u * kNormThreads >= pieces) break;
#pragma unroll
            for (int h = 0; h < static_cast<int>(sizeof(In)) * kPer / 16; ++h)
                w[u][h] = ld_stream(reinterpret_cast<const uint4*>(x + head + (i + u * kNormThreads) * kPer) + h);
        }
#pragma unroll
        for (int u = 0; u < kClipUnroll; ++u) {
            if (i + u * kNormThreads >= pieces) break;
            float v[kPer];
            if constexpr (sizeof(In) == 2) {
                float2 q[4];
                unpack8(w[u][0], q);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[2 * j] = q[j].x * f.factor;
                    v[2 * j + 1] = q[j].y * f.factor;
                }
            } else {
#pragma unroll
                for (int h = 0; h < kPer / 4; ++h) {
                    v[4 * h] = __uint_as_float(w[u][h].x) * f.factor;
                    v[4 * h + 1] = __uint_as_float(w[u][h].y) * f.factor;
                    v[4 * h + 2] = __uint_as_float(w[u][h].z) * f.factor;
                    v[4 * h + 3] = __uint_as_float(w[u][h].w) * f.factor;
                }
            }
            uint4* to = reinterpret_cast<uint4*>(y + head + (i + u * kNormThreads) * kPer);
            if constexpr (sizeof(Out) == 2) {
                st_stream(to, make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])));
            } else {
#pragma unroll
                for (int h = 0; h < kPer / 4; ++h)
                    st_stream(to + h, make_uint4(__float_as_uint(v[4 * h]), __float_as_uint(v[4 * h + 1]),
                                                 __float_as_uint(v[4 * h + 2]), __float_as_uint(v[4 * h + 3])));
            }
        }
    }
    auto one = [&](int i) {
        const float v = as_float(x[i]) * f.factor;
        if constexpr (sizeof(Out) == 2) y[i] = __float2bfloat16_rn(v);
        else y[i] = v;
    };
    if (static_cast<int>(threadIdx.x) < head) one(threadIdx.x);
    if (tail + static_cast<int>(threadIdx.x) < n) one(tail + threadIdx.x);
}

template <int N>
__global__ void __launch_bounds__(kNormThreads, 4) clip_grads_kernel(const __grid_constant__ GradNormParams<N> p)
{
    griddep_launch_dependents();
    const int b = p.blocks - 1 - static_cast<int>(blockIdx.x);
    const GradTensor& t = p.t[norm_tensor_of(p, b)];
    griddep_wait();
    const float norm = __ldcg(p.norm);
    const ClipFactor factor = clip_factor(norm, p.max_norm, p.eps);
    if (factor.factor == 1.0f && t.in == t.out && t.in32 == t.out32) return;
    {
        const int64_t at = static_cast<int64_t>(b - t.first_block) * kNormBlock;
        const int n = static_cast<int>(min(t.numel - at, static_cast<int64_t>(kNormBlock)));
        const float* x32 = static_cast<const float*>(t.in) + at;
        const __nv_bfloat16* x16 = static_cast<const __nv_bfloat16*>(t.in) + at;
        float* y32 = static_cast<float*>(t.out) + at;
        __nv_bfloat16* y16 = static_cast<__nv_bfloat16*>(t.out) + at;
        if (t.in32) {
            if (t.out32) block_scale(x32, y32, n, factor);
            else block_scale(x32, y16, n, factor);
        } else {
            if (t.out32) block_scale(x16, y32, n, factor);
            else block_scale(x16, y16, n, factor);
        }
    }
}

struct GradNormCall {
    const void* const* in;
    void* const* out;            // NULL: the norm alone
    const int64_t* numel;
    const int32_t* in_dtype;
    const int32_t* out_dtype;
    int64_t count;
};

// Fills a launch's descriptors from tensor `first` on; returns how many tensors it took.  Empty ones are passed by.
template <int N>
static int64_t norm_fill(GradNormParams<N>& p, const GradNormCall& c, int64_t first)
{
    p.count = p.blocks = 0;
    int64_t i = first;
    for (; i < c.count && p.count < N; ++i) {
        if (c.numel[i] == 0) continue;
        const int64_t blocks = (c.numel[i] + kNormBlock - 1) / kNormBlock;
        if (blocks > 0x7FFFFFFF - p.blocks) break;
        GradTensor& t = p.t[p.count++];
        t.in = c.in[i];
        t.out = c.out ? c.out[i] : nullptr;
        t.numel = c.numel[i];
        t.in32 = c.in_dtype[i] == MXFP4_OUT_FP32;
        t.out32 = c.out && c.out_dtype[i] == MXFP4_OUT_FP32;
        t.first_block = p.blocks;
        p.blocks += static_cast<int32_t>(blocks);
    }
    return i - first;
}

static int64_t norm_launches(int64_t count) { return (count + kNormMostTensors - 1) / kNormMostTensors; }

template <int N>
static int norm_run(const GradNormCall& c, float max_norm, float eps, float* norm, double* parts, cudaStream_t st)
{
    GradNormParams<N> p;
    memset(&p, 0, offsetof(GradNormParams<N>, t));
    p.norm = norm;
    p.max_norm = max_norm;
    p.eps = eps;
    int64_t launches = 0;
    for (int64_t i = 0; i < c.count;) {
        i += norm_fill(p, c, i);
        p.parts = parts + launches++ * kNormCtas;
        if (launch_kernel_pdl(grad_norm_kernel<N>, kNormCtas, kNormThreads, 0, st, p) != cudaSuccess) return MXFP4_ERR_CUDA;
    }
    if (launch_kernel_pdl(grad_norm_join_kernel, 1, kNormThreads, 0, st, parts, static_cast<int>(launches * kNormCtas), norm) !=
        cudaSuccess)
        return MXFP4_ERR_CUDA;
    for (int64_t i = 0; c.out && i < c.count;) {
        i += norm_fill(p, c, i);
        if (p.blocks == 0) continue;
        if (launch_kernel_pdl(clip_grads_kernel<N>, p.blocks, kNormThreads, 0, st, p) != cudaSuccess) return MXFP4_ERR_CUDA;
    }
    return MXFP4_OK;
}

// Whether an output overlaps another tensor of the call.
struct GradSpan {
    uintptr_t begin, end;
    bool written;
};

static int norm_overlap(const GradNormCall& c)
{
    GradSpan* s = static_cast<GradSpan*>(malloc(sizeof(GradSpan) * 2 * static_cast<size_t>(c.count)));
    if (!s) return MXFP4_ERR_WORKSPACE;
    size_t n = 0;
    for (int64_t i = 0; i < c.count; ++i) {
        if (c.numel[i] == 0) continue;
        const uintptr_t a = reinterpret_cast<uintptr_t>(c.in[i]), b = reinterpret_cast<uintptr_t>(c.out[i]);
        s[n++] = {b, b + c.numel[i] * (c.out_dtype[i] == MXFP4_OUT_FP32 ? 4u : 2u), true};
        if (a != b || c.in_dtype[i] != c.out_dtype[i])
            s[n++] = {a, a + c.numel[i] * (c.in_dtype[i] == MXFP4_OUT_FP32 ? 4u : 2u), false};
    }
    std::sort(s, s + n, [](const GradSpan& x, const GradSpan& y) { return x.begin < y.begin; });
    uintptr_t all = 0, written = 0;    // ends of what began so far, and of what of it is written
    int rc = MXFP4_OK;
    for (size_t i = 0; i < n && rc == MXFP4_OK; ++i) {
        if (s[i].begin < (s[i].written ? all : written)) rc = MXFP4_ERR_SHAPE;
        if (s[i].end > all) all = s[i].end;
        if (s[i].written && s[i].end > written) written = s[i].end;
    }
    free(s);
    return rc;
}

int grad_norm_take_status(int* status) { return take_unit_status(status); }
int grad_norm_selftest(cudaStream_t st) { return unit_selftest(st); }

}  // namespace mxfp4

using namespace mxfp4;

extern "C" {

size_t mxfp4_grad_norm_workspace_bytes(int64_t count)
{
    if (count <= 0 || count > 0x3FFFFFFF) return 0;
    return static_cast<size_t>(norm_launches(count)) * kNormCtas * sizeof(double);
}

static int norm_call(const GradNormCall& c, float max_norm, float eps, float* norm, void* workspace, size_t workspace_bytes,
                     void* stream)
{
    if (c.count <= 0 || c.count > 0x3FFFFFFF) return MXFP4_ERR_SHAPE;
    for (int64_t i = 0; i < c.count; ++i) {
        if (c.numel[i] < 0 || c.numel[i] > (int64_t{1} << 44)) return MXFP4_ERR_SHAPE;
        for (int o = 0; o < (c.out ? 2 : 1); ++o) {
            const int type = o ? c.out_dtype[i] : c.in_dtype[i];
            const void* ptr = o ? c.out[i] : c.in[i];
            if (type != MXFP4_OUT_BF16 && type != MXFP4_OUT_FP32) return MXFP4_ERR_ENUM;
            if (c.numel[i] > 0 && !ptr) return MXFP4_ERR_NULL;
            if ((reinterpret_cast<uintptr_t>(ptr) & (type == MXFP4_OUT_FP32 ? 3u : 1u)) != 0) return MXFP4_ERR_ALIGN;
        }
    }
    int rc = MXFP4_OK;
    if (c.out && (rc = norm_overlap(c)) != MXFP4_OK) return rc;
    if (!workspace || workspace_bytes < mxfp4_grad_norm_workspace_bytes(c.count)) return MXFP4_ERR_WORKSPACE;
    if (!aligned16(workspace) || (reinterpret_cast<uintptr_t>(norm) & 3u)) return MXFP4_ERR_ALIGN;
    if ((rc = device_status_code(device_info())) != MXFP4_OK) return rc;
    double* parts = static_cast<double*>(workspace);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    // a launch's arguments are copied when it is queued: as few as the call needs
    if (c.count <= 16) return norm_run<16>(c, max_norm, eps, norm, parts, st);
    if (c.count <= 128) return norm_run<128>(c, max_norm, eps, norm, parts, st);
    return norm_run<kNormMostTensors>(c, max_norm, eps, norm, parts, st);
}

int mxfp4_grad_norm(const void* const* tensors, const int64_t* numel, const int32_t* dtypes, int64_t count, float* norm,
                    void* workspace, size_t workspace_bytes, void* stream)
{
    if (!tensors || !numel || !dtypes || !norm) return MXFP4_ERR_NULL;
    const GradNormCall c = {tensors, nullptr, numel, dtypes, nullptr, count};
    return norm_call(c, 0.0f, 0.0f, norm, workspace, workspace_bytes, stream);
}

int mxfp4_clip_grads(const void* const* tensors, const int64_t* numel, const int32_t* dtypes, int64_t count, float max_norm,
                     float eps, void* const* out, const int32_t* out_dtypes, float* norm, void* workspace,
                     size_t workspace_bytes, void* stream)
{
    if (!tensors || !numel || !dtypes || !out || !out_dtypes || !norm) return MXFP4_ERR_NULL;
    if (!(max_norm >= 0.0f) || !(eps >= 0.0f) || isinf(eps)) return MXFP4_ERR_ENUM;
    const GradNormCall c = {tensors, out, numel, dtypes, out_dtypes, count};
    return norm_call(c, max_norm, eps, norm, workspace, workspace_bytes, stream);
}

}  // extern "C"
