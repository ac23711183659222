// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and the
// gradient with respect to the logits.
//
// Forward: one pass over the logits.  A thread keeps a reference m, S = sum 2^a and A = sum a 2^a
// with a = (x - m) * scale * log2(e) over its vectors; at the end the CTA brings all threads to a
// common m, and then
//     lse = scale * m + ln S,   entropy = ln S - ln 2 * A / S.
// The reference is the thread's first maximum and moves only when a later one is more than a factor
// of 2^8 above it, so the sums are hardly ever rescaled on the way (a running maximum would make
// some lane of a warp rescale at most vectors), and what the late step back to a common
// reference can cost in precision stays within 8 * 2^-24 of a nat.
//
// Top alternatives: every thread remembers its largest logit and the first vector that held it.
// The top_k-th best of those is a lower bound for the row's top_k-th best logit that exactly top_k
// threads reach, so only their vectors are looked at again (they are still in L2), and what
// reaches the bound -- a few dozen logits -- is ranked in shared memory.
//
// A row is split over several CTAs when there are too few rows to fill the device; each split
// leaves (m, S, A) and its own alternatives in the workspace and a second kernel joins them.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/mxfp4.h"
#include "host_common.cuh"
#include "ptx_sm100.cuh"
#include "row_io.cuh"
#include "tma_host.cuh"

namespace mxfp4 {

constexpr int kLpThreads = 512;
constexpr int kLpMaxTop = 32;
constexpr int kLpCandidates = 1024;          // ranked in shared memory; more take the slow way
constexpr int kLpFillCtas = 296;             // two per SM of the device the kernel is tuned on
constexpr int kLpMaxSplits = 74;
constexpr float kLpReach = 8.0f;             // see above
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <class T>
struct LogitVec;
template <>
struct LogitVec<__nv_bfloat16> {
    static constexpr int kN = 8;
    static constexpr int kKeyShift = 16;     // the low half of a bf16 value's key is constant
    static __device__ __forceinline__ void get(const uint4& w, float (&v)[8])
    {
        v[0] = bf16_lo(w.x); v[1] = bf16_hi(w.x);
        v[2] = bf16_lo(w.y); v[3] = bf16_hi(w.y);
        v[4] = bf16_lo(w.z); v[5] = bf16_hi(w.z);
        v[6] = bf16_lo(w.w); v[7] = bf16_hi(w.w);
    }
    static __device__ __forceinline__ uint4 put(const float (&v)[8])
    {
        return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    }
    static __device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
    static __device__ __forceinline__ void set(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
};
template <>
struct LogitVec<float> {
    static constexpr int kN = 4;
    static constexpr int kKeyShift = 0;
    static __device__ __forceinline__ void get(const uint4& w, float (&v)[4])
    {
        v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y);
        v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
    }
    static __device__ __forceinline__ uint4 put(const float (&v)[4])
    {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
    static __device__ __forceinline__ float one(const float* p) { return *p; }
    static __device__ __forceinline__ void set(float* p, float v) { *p = v; }
};

__device__ __forceinline__ float exp2_approx(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// larger of the two, NaN if either is
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Unsigned key that orders fp32 values (both zeros are one value); 0 stands for "none", which is
// also what -infinity and NaN get.
__device__ __forceinline__ uint32_t order_key(float x)
{
    if (!(x > -INFINITY)) return 0u;
    const uint32_t b = __float_as_uint(x + 0.0f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k)
{
    return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k);
}
// value first, then lowest index
__device__ __forceinline__ uint64_t full_key(float x, uint32_t index)
{
    const uint32_t k = order_key(x);
    return k ? (static_cast<uint64_t>(k) << 32) | (0xFFFFFFFFu - index) : 0ull;
}

struct LogprobsParams {
    const void* logits;
    const int64_t* targets;
    int64_t ld;
    int64_t tokens;
    int32_t vocab;
    int32_t top_k;
    int32_t splits;
    int32_t vecs_per_split;
    float scale;
    float* logp;
    float* entropy;
    float* lse;
    float* top_logp;
    int64_t* top_index;
    float4* part_sums;          // [row][split]: m, S, A
    uint64_t* part_keys;        // [row][split][top_k]
};

// (m, S, A) of part of a row
struct SoftSums {
    float m, s, a;
};

// The sums of two parts relative to a common reference.  An empty part (m = -infinity) adds nothing
// but what a NaN left in its s.
__device__ __forceinline__ SoftSums rebase(const SoftSums& v, float m, float c)
{
    if (m == -INFINITY) return {m, v.s, v.a};
    const float d = fmaxf((v.m - m) * c, -1000.0f);
    const float f = exp2_approx(d);
    return {m, v.s * f, f * fmaf(d, v.s, v.a)};
}

__device__ __forceinline__ SoftSums warp_join(SoftSums v, float c)
{
    float m = v.m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    v = rebase(v, m, c);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        v.s += __shfl_xor_sync(0xffffffffu, v.s, o);
        v.a += __shfl_xor_sync(0xffffffffu, v.a, o);
    }
    return v;
}

// Over the CTA; every thread gets the result.  Ends with every thread past a barrier.
__device__ __forceinline__ SoftSums block_join(SoftSums v, float c, SoftSums* red)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    v = warp_join(v, c);
    if (lane == 0) red[warp] = v;
    __syncthreads();
    v = lane < static_cast<int>(blockDim.x >> 5) ? red[lane] : SoftSums{-INFINITY, 0.0f, 0.0f};
    return warp_join(v, c);
}

// Row results of one thread.
__device__ __forceinline__ float finish_row(const LogprobsParams& p, int64_t row, const SoftSums& v)
{
    if (v.m == -INFINITY && v.s == 0.0f) {           // nothing but masked logits
        p.lse[row] = -INFINITY;
        if (p.entropy) p.entropy[row] = 0.0f;
        return -INFINITY;
    }
    const float log_s = kLn2 * log2f(v.s);
    const float lse = v.m == -INFINITY ? v.s : fmaf(v.m, p.scale, log_s);
    p.lse[row] = lse;
    if (p.entropy) p.entropy[row] = v.m == -INFINITY ? v.s : log_s - kLn2 * (v.a / v.s);
    return lse;
}

template <class T>
__device__ __forceinline__ void finish_target(const LogprobsParams& p, int64_t row, float lse)
{
    if (!p.logp) return;
    const int64_t t = p.targets[row];
    float r = 0.0f;
    if (t >= p.vocab) {
        r = NAN;
    } else if (t >= 0) {
        const float x = LogitVec<T>::one(static_cast<const T*>(p.logits) + row * p.ld + t);
        r = lse == -INFINITY ? -INFINITY : fmaf(x, p.scale, -lse);
    }
    p.logp[row] = r;
}

__device__ __forceinline__ void write_top(const LogprobsParams& p, int64_t row, int rank, uint64_t key, float lse)
{
    const int64_t at = row * p.top_k + rank;
    const bool bad = lse != lse;
    const bool none = bad || key == 0ull;
    p.top_logp[at] = bad ? NAN : none ? -INFINITY : fmaf(key_value(static_cast<uint32_t>(key >> 32)), p.scale, -lse);
    p.top_index[at] = none ? -1 : static_cast<int64_t>(0xFFFFFFFFu - static_cast<uint32_t>(key));
}

// The largest key that at least `want` threads' keys (one per thread, compared above `low` bits)
// reach; 0 when fewer than `want` threads have one.
__device__ __forceinline__ uint32_t block_kth(uint32_t key, int want, int low)
{
    uint32_t found = 0;
    for (int b = 31; b >= low; --b) {
        const uint32_t probe = found | (1u << b);
        if (__syncthreads_count(key >= probe) >= want) found = probe;
    }
    return found;
}

struct TopScratch {
    uint64_t keys[kLpCandidates];
    uint64_t best;
    int32_t owner[kLpMaxTop];
    int32_t owners;
    int32_t n;
};

// The elements of a row a CTA owns: vectors first .. first + count, and the unaligned head or tail.
template <class T>
struct RowPart {
    const T* row;
    int head;                  // elements before the first 16-byte boundary
    int first, count;          // vectors
    int loose0, n_loose0;      // single elements: at the row's head,
    int loose1, n_loose1;      // and at its end
    __device__ __forceinline__ int loose_index(int i) const { return i < n_loose0 ? loose0 + i : loose1 + i - n_loose0; }
    __device__ __forceinline__ const T* vec(int v) const { return row + head + static_cast<int64_t>(v) * LogitVec<T>::kN; }
};

template <class T>
__device__ __forceinline__ RowPart<T> row_part(const LogprobsParams& p, int64_t row, int split)
{
    constexpr int kN = LogitVec<T>::kN;
    RowPart<T> r;
    r.row = static_cast<const T*>(p.logits) + row * p.ld;
    const int off = static_cast<int>(reinterpret_cast<uintptr_t>(r.row) & 15u) / static_cast<int>(sizeof(T));
    r.head = off ? min(kN - off, p.vocab) : 0;
    const int vecs = (p.vocab - r.head) / kN;
    r.first = min(split * p.vecs_per_split, vecs);
    r.count = min(p.vecs_per_split, vecs - r.first);
    r.loose0 = 0;
    r.n_loose0 = split == 0 ? r.head : 0;
    r.loose1 = r.head + vecs * kN;
    r.n_loose1 = split == p.splits - 1 ? p.vocab - r.loose1 : 0;
    return r;
}

// The part's `top_k` best keys in descending order; `emit(rank, key)` is called once for every rank
// that exists.  `best` / `best_vec`: the thread's largest logit and the first vector with it.
template <class T, class Emit>
__device__ __forceinline__ void block_top(const RowPart<T>& part, int top_k, float best, int best_vec, TopScratch& sc,
                                          Emit emit)
{
    constexpr int kN = LogitVec<T>::kN;
    const int tid = threadIdx.x;
    if (tid == 0) sc.owners = sc.n = 0;
    // bound: value, then vector (all keys of threads that have one differ in the pair)
    const uint32_t key = order_key(best);
    const uint32_t kth = block_kth(key, top_k, LogitVec<T>::kKeyShift);
    // bf16 keys of negative values end in ones: the bound found above has zeros there
    const bool above = key != 0u && (key >> LogitVec<T>::kKeyShift) > (kth >> LogitVec<T>::kKeyShift);
    const bool equal = key != 0u && (key >> LogitVec<T>::kKeyShift) == (kth >> LogitVec<T>::kKeyShift);
    const int n_above = __syncthreads_count(above);
    const int n_equal = __syncthreads_count(equal);
    uint32_t vec_key = 0u;                      // of the vectors with a value equal to the bound: the first ones
    if (n_above + n_equal > top_k)
        vec_key = block_kth(equal ? 0x7FFFFFFFu - static_cast<uint32_t>(best_vec) : 0u, top_k - n_above, 0);
    if (above || (equal && 0x7FFFFFFFu - static_cast<uint32_t>(best_vec) >= vec_key))
        sc.owner[atomicAdd(&sc.owners, 1)] = tid;
    __syncthreads();
    auto take = [&](float x, uint32_t index) {
        const uint64_t k = full_key(x, index);
        if (k == 0ull) return;
        const int at = atomicAdd(&sc.n, 1);
        if (at < kLpCandidates) sc.keys[at] = k;
    };
    // the owners' vectors again, one warp per owner, a lane per vector
    const int lane = tid & 31;
    for (int o = tid >> 5; o < sc.owners; o += kLpThreads / 32) {
        for (int v = sc.owner[o] + lane * kLpThreads; v < part.count; v += 32 * kLpThreads) {
            const T* at = part.vec(part.first + v);
            float x[kN];
            LogitVec<T>::get(*reinterpret_cast<const uint4*>(at), x);
            const bool late = 0x7FFFFFFFu - static_cast<uint32_t>(part.first + v) < vec_key;
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                const uint32_t k = order_key(x[i]) >> LogitVec<T>::kKeyShift, b = kth >> LogitVec<T>::kKeyShift;
                if (k > b || (k == b && !late)) take(x[i], static_cast<uint32_t>(at - part.row) + i);
            }
        }
    }
    for (int i = tid; i < part.n_loose0 + part.n_loose1; i += kLpThreads) {
        const int at = part.loose_index(i);
        take(LogitVec<T>::one(part.row + at), static_cast<uint32_t>(at));
    }
    __syncthreads();
    const int n = sc.n;
    if (n <= kLpCandidates) {
        for (int i = tid; i < n; i += kLpThreads) {
            const uint64_t k = sc.keys[i];
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += sc.keys[j] > k;
            if (rank < top_k) emit(rank, k);
        }
    } else {
        // thousands of logits above the bound: rank after rank, each from the whole part
        uint64_t last = ~0ull;
        for (int rank = 0; rank < top_k; ++rank) {
            if (tid == 0) sc.best = 0ull;
            __syncthreads();
            uint64_t mine = 0ull;
            auto look = [&](float x, uint32_t index) {
                const uint64_t k = full_key(x, index);
                if (k < last && k > mine) mine = k;
            };
            for (int v = tid; v < part.count; v += kLpThreads) {
                const T* at = part.vec(part.first + v);
                float x[kN];
                LogitVec<T>::get(*reinterpret_cast<const uint4*>(at), x);
#pragma unroll
                for (int i = 0; i < kN; ++i) look(x[i], static_cast<uint32_t>(at - part.row) + i);
            }
            for (int i = tid; i < part.n_loose0 + part.n_loose1; i += kLpThreads)
                look(LogitVec<T>::one(part.row + part.loose_index(i)), static_cast<uint32_t>(part.loose_index(i)));
            atomicMax(reinterpret_cast<unsigned long long*>(&sc.best), static_cast<unsigned long long>(mine));
            __syncthreads();
            last = sc.best;
            if (tid == 0 && last) emit(rank, last);
            __syncthreads();
            if (last == 0ull) break;
        }
    }
}

template <class T, bool TOP>
__global__ void __launch_bounds__(kLpThreads, 2) logprobs_forward_kernel(const LogprobsParams p)
{
    constexpr int kN = LogitVec<T>::kN;
    __shared__ SoftSums red[kLpThreads / 32];
    __shared__ TopScratch scratch;
    griddep_launch_dependents();
    griddep_wait();
    const int64_t row = blockIdx.x / p.splits;
    const int split = blockIdx.x % p.splits;
    const RowPart<T> part = row_part<T>(p, row, split);
    const float c = p.scale * kLog2e;
    const float reach = kLpReach / c;

    float m = -INFINITY, limit = -INFINITY, ref = 0.0f;   // ref = m, or 0 while nothing but masked logits came
    float2 s = make_float2(0.0f, 0.0f), a = make_float2(0.0f, 0.0f);
    float best = -INFINITY;
    int best_vec = 0;
    auto add = [&](const float* x, int n) {               // n even, or 1
        float top = x[0];
        for (int i = 1; i < n; ++i) top = fmaxf(top, x[i]);
        if (top > limit) {
            if (m > -INFINITY) {
                const float d = fmaxf((m - top) * c, -1000.0f), f = exp2_approx(d);
                a.x = f * fmaf(d, s.x, a.x);
                a.y = f * fmaf(d, s.y, a.y);
                s.x *= f;
                s.y *= f;
            }
            m = ref = top;
            limit = top + reach;
        }
        return top;
    };
    auto accumulate = [&](const float (&x)[kN], int vec) {
        const float top = add(x, kN);
        if (TOP && top > best) {
            best = top;
            best_vec = vec;
        }
#pragma unroll
        for (int i = 0; i < kN; i += 2) {
            float2 d = __fadd2_rn(make_float2(x[i], x[i + 1]), make_float2(-ref, -ref));
            d = __fmul2_rn(d, make_float2(c, c));
            d.x = max_nan(d.x, -300.0f);                // a masked logit: 2^-300 = 0, and 0 * -300 is 0
            d.y = max_nan(d.y, -300.0f);
            const float2 e = make_float2(exp2_approx(d.x), exp2_approx(d.y));
            s = __fadd2_rn(s, e);
            a = __ffma2_rn(d, e, a);
        }
    };
    const T* base = part.vec(part.first);
    constexpr int kUnroll = 4;
    int v = threadIdx.x;
    for (; v + (kUnroll - 1) * kLpThreads < part.count; v += kUnroll * kLpThreads) {
        uint4 w[kUnroll];
#pragma unroll
        for (int j = 0; j < kUnroll; ++j) w[j] = ld_stream(base + static_cast<int64_t>(v + j * kLpThreads) * kN);
#pragma unroll
        for (int j = 0; j < kUnroll; ++j) {
            float x[kN];
            LogitVec<T>::get(w[j], x);
            accumulate(x, part.first + v + j * kLpThreads);
        }
    }
    for (; v < part.count; v += kLpThreads) {
        float x[kN];
        LogitVec<T>::get(ld_stream(base + static_cast<int64_t>(v) * kN), x);
        accumulate(x, part.first + v);
    }
    if (static_cast<int>(threadIdx.x) < part.n_loose0 + part.n_loose1) {
        const float x = LogitVec<T>::one(part.row + part.loose_index(threadIdx.x));
        add(&x, 1);
        const float d = max_nan((x - ref) * c, -300.0f), e = exp2_approx(d);
        s.x += e;
        a.x = fmaf(d, e, a.x);
    }
    const SoftSums sums = block_join({m, s.x + s.y, a.x + a.y}, c, red);

    if (p.splits == 1) {
        __shared__ float row_lse;
        if (threadIdx.x == 0) {
            const float lse = finish_row(p, row, sums);
            finish_target<T>(p, row, lse);
            row_lse = lse;
        }
        if (TOP) {
            // ranks that do not exist keep this
            __syncthreads();
            const float lse = row_lse;
            if (static_cast<int>(threadIdx.x) < p.top_k) write_top(p, row, threadIdx.x, 0ull, lse);
            __syncthreads();
            if (lse == lse && lse != -INFINITY)
                block_top<T>(part, p.top_k, best, best_vec, scratch,
                             [&](int rank, uint64_t key) { write_top(p, row, rank, key, lse); });
        }
    } else {
        const int64_t at = row * p.splits + split;
        if (threadIdx.x == 0) p.part_sums[at] = make_float4(sums.m, sums.s, sums.a, 0.0f);
        if (TOP) {
            if (static_cast<int>(threadIdx.x) < p.top_k) p.part_keys[at * p.top_k + threadIdx.x] = 0ull;
            __syncthreads();
            block_top<T>(part, p.top_k, best, best_vec, scratch,
                         [&](int rank, uint64_t key) { p.part_keys[at * p.top_k + rank] = key; });
        }
    }
}

// Joins the splits of a row: the sums, and rank after rank the largest key not taken yet.
constexpr int kLpJoinThreads = 256;
template <class T>
__global__ void __launch_bounds__(kLpJoinThreads) logprobs_join_kernel(const LogprobsParams p)
{
    __shared__ SoftSums red[kLpJoinThreads / 32];
    __shared__ uint64_t keys[kLpMaxSplits * kLpMaxTop];
    __shared__ float row_lse;
    griddep_launch_dependents();
    griddep_wait();
    const int64_t row = blockIdx.x;
    const float c = p.scale * kLog2e;
    SoftSums v = {-INFINITY, 0.0f, 0.0f};
    for (int i = threadIdx.x; i < p.splits; i += kLpJoinThreads) {
        const float4 f = p.part_sums[row * p.splits + i];
        const SoftSums w = {f.x, f.y, f.z};
        const float m = fmaxf(v.m, w.m);
        const SoftSums x = rebase(v, m, c), y = rebase(w, m, c);
        v = {m, x.s + y.s, x.a + y.a};
    }
    v = block_join(v, c, red);
    if (threadIdx.x == 0) {
        const float lse = finish_row(p, row, v);
        finish_target<T>(p, row, lse);
        row_lse = lse;
    }
    if (p.top_k == 0) return;
    const int n = p.splits * p.top_k;
    for (int i = threadIdx.x; i < n; i += kLpJoinThreads) keys[i] = p.part_keys[row * n + i];
    __syncthreads();
    const float lse = row_lse;
    if (static_cast<int>(threadIdx.x) < p.top_k) write_top(p, row, threadIdx.x, 0ull, lse);
    __syncthreads();
    if (lse != lse || lse == -INFINITY) return;
    // a key's rank is the number of larger ones; each split's keys are in descending order
    for (int i = threadIdx.x; i < n; i += kLpJoinThreads) {
        const uint64_t k = keys[i];
        if (k == 0ull) continue;
        int rank = i % p.top_k;
        for (int s = 0; s < p.splits && rank < p.top_k; ++s) {
            if (s == i / p.top_k) continue;
            for (int j = 0; j < p.top_k && keys[s * p.top_k + j] > k; ++j) ++rank;
        }
        if (rank < p.top_k) write_top(p, row, rank, k, lse);
    }
}

struct LogprobsGradParams {
    const void* logits;
    void* dlogits;
    const int64_t* targets;
    const float* lse;
    const float* entropy;
    const float* d_logp;
    const float* d_entropy;
    int64_t ld, ld_d;
    int64_t tokens;
    int32_t vocab;
    int32_t parts;               // CTAs per row
    float scale;
};

constexpr int kLpGradThreads = 256;
constexpr int kLpGradVecs = 16;              // 16-byte vectors per thread

template <class T>
__global__ void __launch_bounds__(kLpGradThreads) logprobs_backward_kernel(const LogprobsGradParams p)
{
    constexpr int kN = LogitVec<T>::kN;
    griddep_launch_dependents();
    griddep_wait();
    const int64_t row = blockIdx.x / p.parts;
    const int part = blockIdx.x % p.parts;
    const T* src = static_cast<const T*>(p.logits) + row * p.ld;
    T* dst = static_cast<T*>(p.dlogits) + row * p.ld_d;
    const int64_t target = p.targets ? p.targets[row] : -1;
    const float lse = p.lse[row];
    float gl = p.d_logp && target >= 0 ? p.d_logp[row] : 0.0f;
    if (p.d_logp && target >= p.vocab) gl = NAN;
    const float ge = p.d_entropy ? p.d_entropy[row] : 0.0f;
    const float base = fmaf(ge, p.entropy && p.d_entropy ? p.entropy[row] : 0.0f, gl);
    const bool zero = (gl == 0.0f && ge == 0.0f) || lse == -INFINITY;
    // the gradient without the target's own term: -scale * p * (base + ge * (z - lse))
    auto grad = [&](float x, int index) {
        const float l = fmaf(x, p.scale, -lse);
        const float lc = max_nan(l, -300.0f);                 // masked: p = 0, and 0 * -300 is 0
        const float q = exp2_approx(lc * kLog2e);
        float g = -q * fmaf(ge, lc, base);
        if (index == target) g += gl;
        return g * p.scale;
    };
    const int off_s = static_cast<int>(reinterpret_cast<uintptr_t>(src) & 15u);
    const int off_d = static_cast<int>(reinterpret_cast<uintptr_t>(dst) & 15u);
    const int per = kLpGradThreads * kLpGradVecs * kN;          // elements a CTA handles
    if (off_s == off_d) {
        const int head = off_s ? min(kN - off_s / static_cast<int>(sizeof(T)), p.vocab) : 0;
        const int vecs = (p.vocab - head) / kN;
        const int first = part * (kLpGradThreads * kLpGradVecs);
        const int last = min(first + kLpGradThreads * kLpGradVecs, vecs);
        if (zero) {
            for (int v = first + threadIdx.x; v < last; v += kLpGradThreads)
                st_stream(dst + head + static_cast<int64_t>(v) * kN, make_uint4(0u, 0u, 0u, 0u));
        } else {
            constexpr int kUnroll = 4;
            for (int v = first + threadIdx.x; v < last; v += kUnroll * kLpGradThreads) {
                uint4 w[kUnroll];
#pragma unroll
                for (int j = 0; j < kUnroll; ++j)
                    if (v + j * kLpGradThreads < last)
                        w[j] = ld_stream(src + head + static_cast<int64_t>(v + j * kLpGradThreads) * kN);
#pragma unroll
                for (int j = 0; j < kUnroll; ++j) {
                    const int at = head + (v + j * kLpGradThreads) * kN;
                    if (v + j * kLpGradThreads < last) {
                        float x[kN];
                        LogitVec<T>::get(w[j], x);
#pragma unroll
                        for (int i = 0; i < kN; ++i) x[i] = grad(x[i], at + i);
                        st_stream(dst + at, LogitVec<T>::put(x));
                    }
                }
            }
        }
        // the unaligned ends of the row
        if (part == 0 && static_cast<int>(threadIdx.x) < head)
            LogitVec<T>::set(dst + threadIdx.x, zero ? 0.0f : grad(LogitVec<T>::one(src + threadIdx.x), threadIdx.x));
        const int tail = head + vecs * kN + static_cast<int>(threadIdx.x);
        if (part == p.parts - 1 && tail < p.vocab && static_cast<int>(threadIdx.x) < kN)
            LogitVec<T>::set(dst + tail, zero ? 0.0f : grad(LogitVec<T>::one(src + tail), tail));
    } else {
        // the two rows start at different offsets inside 16 bytes: element by element
        for (int64_t i = static_cast<int64_t>(part) * per + threadIdx.x;
             i < p.vocab && i < static_cast<int64_t>(part + 1) * per; i += kLpGradThreads)
            LogitVec<T>::set(dst + i, zero ? 0.0f : grad(LogitVec<T>::one(src + i), static_cast<int>(i)));
    }
}

// Splits per row: enough CTAs to fill the device, but at least one vector per thread in each.
// Eight-element vectors are assumed for both types, so that the size does not depend on the type.
static int logprobs_splits(int64_t tokens, int64_t vocab)
{
    const int64_t by_fill = (kLpFillCtas + tokens - 1) / tokens;
    const int64_t by_work = (vocab / 8 + kLpThreads - 1) / kLpThreads;
    int64_t s = by_fill < by_work ? by_fill : by_work;
    if (s > kLpMaxSplits) s = kLpMaxSplits;
    return static_cast<int>(s < 1 ? 1 : s);
}

static int logprobs_shape_ok(const void* logits, int dtype, int64_t tokens, int64_t vocab, int64_t ld, float scale)
{
    if (!logits) return MXFP4_ERR_NULL;
    if (dtype != MXFP4_OUT_BF16 && dtype != MXFP4_OUT_FP32) return MXFP4_ERR_ENUM;
    if (!(scale > 0.0f) || !(scale <= 3.4e38f)) return MXFP4_ERR_ENUM;
    if (tokens <= 0 || vocab <= 0 || ld < vocab) return MXFP4_ERR_SHAPE;
    if (vocab > 0x3FFFFFFF || tokens > 0x7FFFFFFF / (kLpFillCtas + 1)) return MXFP4_ERR_SHAPE;
    if (reinterpret_cast<uintptr_t>(logits) & (dtype == MXFP4_OUT_BF16 ? 1u : 3u)) return MXFP4_ERR_ALIGN;
    return MXFP4_OK;
}

template <class T>
static int launch_logprobs_forward(const LogprobsParams& p, cudaStream_t st)
{
    const int grid = static_cast<int>(p.tokens * p.splits);
    const cudaError_t e = p.top_k > 0
                              ? launch_kernel_pdl(logprobs_forward_kernel<T, true>, grid, kLpThreads, 0, st, p)
                              : launch_kernel_pdl(logprobs_forward_kernel<T, false>, grid, kLpThreads, 0, st, p);
    if (e != cudaSuccess) return MXFP4_ERR_CUDA;
    if (p.splits > 1 && launch_kernel_pdl(logprobs_join_kernel<T>, static_cast<int>(p.tokens), kLpJoinThreads, 0, st,
                                          p) != cudaSuccess)
        return MXFP4_ERR_CUDA;
    return MXFP4_OK;
}

}  // namespace mxfp4

using namespace mxfp4;

extern "C" {

size_t mxfp4_logprobs_workspace_bytes(int64_t tokens, int64_t vocab, int top_k)
{
    if (tokens <= 0 || vocab <= 0 || top_k < 0 || top_k > kLpMaxTop) return 0;
    const int64_t splits = logprobs_splits(tokens, vocab);
    if (splits == 1) return 0;
    return static_cast<size_t>(tokens * splits) * (sizeof(float4) + static_cast<size_t>(top_k) * sizeof(uint64_t));
}

int mxfp4_logprobs_forward(const void* logits, int dtype, int64_t tokens, int64_t vocab, int64_t ld,
                           const int64_t* targets, float scale, float* logp, float* entropy, float* lse, int top_k,
                           float* top_logp, int64_t* top_index, void* workspace, size_t workspace_bytes, void* stream)
{
    int rc = logprobs_shape_ok(logits, dtype, tokens, vocab, ld, scale);
    if (rc != MXFP4_OK) return rc;
    if (!lse || (targets != nullptr) != (logp != nullptr)) return MXFP4_ERR_NULL;
    if (top_k < 0 || top_k > kLpMaxTop) return MXFP4_ERR_ENUM;
    if (top_k > 0 && (!top_logp || !top_index)) return MXFP4_ERR_NULL;
    const size_t need = mxfp4_logprobs_workspace_bytes(tokens, vocab, top_k);
    if (need > 0 && (!workspace || workspace_bytes < need)) return MXFP4_ERR_WORKSPACE;
    if (need > 0 && !aligned16(workspace)) return MXFP4_ERR_ALIGN;
    const DeviceInfo& dev = device_info();
    if ((rc = device_status_code(dev)) != MXFP4_OK) return rc;
    LogprobsParams p;
    p.logits = logits;
    p.targets = targets;
    p.ld = ld;
    p.tokens = tokens;
    p.vocab = static_cast<int32_t>(vocab);
    p.top_k = top_k;
    p.splits = logprobs_splits(tokens, vocab);
    const int64_t vecs = vocab / (dtype == MXFP4_OUT_BF16 ? 8 : 4);
    p.vecs_per_split = static_cast<int32_t>((vecs + p.splits - 1) / p.splits);
    p.scale = scale;
    p.logp = logp;
    p.entropy = entropy;
    p.lse = lse;
    p.top_logp = top_logp;
    p.top_index = top_index;
    p.part_sums = static_cast<float4*>(workspace);
    p.part_keys = need ? reinterpret_cast<uint64_t*>(p.part_sums + tokens * p.splits) : nullptr;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dtype == MXFP4_OUT_BF16 ? launch_logprobs_forward<__nv_bfloat16>(p, st)
                                   : launch_logprobs_forward<float>(p, st);
}

int mxfp4_logprobs_backward(const void* logits, int dtype, int64_t tokens, int64_t vocab, int64_t ld,
                            const int64_t* targets, float scale, const float* lse, const float* entropy,
                            const float* d_logp, const float* d_entropy, void* dlogits, int64_t ld_d, void* stream)
{
    int rc = logprobs_shape_ok(logits, dtype, tokens, vocab, ld, scale);
    if (rc != MXFP4_OK) return rc;
    if (!lse || !dlogits || (d_logp && !targets) || (d_entropy && !entropy)) return MXFP4_ERR_NULL;
    if (ld_d < vocab) return MXFP4_ERR_SHAPE;
    if (reinterpret_cast<uintptr_t>(dlogits) & (dtype == MXFP4_OUT_BF16 ? 1u : 3u)) return MXFP4_ERR_ALIGN;
    const int64_t per = kLpGradThreads * kLpGradVecs * (dtype == MXFP4_OUT_BF16 ? 8 : 4);
    const int64_t parts = (vocab + per - 1) / per;
    if (tokens > 0x7FFFFFFF / parts) return MXFP4_ERR_SHAPE;
    const DeviceInfo& dev = device_info();
    if ((rc = device_status_code(dev)) != MXFP4_OK) return rc;
    LogprobsGradParams p;
    p.logits = logits;
    p.dlogits = dlogits;
    p.targets = targets;
    p.lse = lse;
    p.entropy = entropy;
    p.d_logp = d_logp;
    p.d_entropy = d_entropy;
    p.ld = ld;
    p.ld_d = ld_d;
    p.tokens = tokens;
    p.vocab = static_cast<int32_t>(vocab);
    p.parts = static_cast<int32_t>(parts);
    p.scale = scale;
    const int grid = static_cast<int>(tokens * parts);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e =
        dtype == MXFP4_OUT_BF16 ? launch_kernel_pdl(logprobs_backward_kernel<__nv_bfloat16>, grid, kLpGradThreads, 0, st, p)
                                : launch_kernel_pdl(logprobs_backward_kernel<float>, grid, kLpGradThreads, 0, st, p);
    return e == cudaSuccess ? MXFP4_OK : MXFP4_ERR_CUDA;
}

}  // extern "C"
