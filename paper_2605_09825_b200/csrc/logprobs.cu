// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and the
// gradient with respect to the logits.
//
// Forward: one pass over the logits.  A thread keeps a reference m, S = sum 2^a and A = sum a 2^a
// with a = (x - m) * scale * log2(e) over its vectors; at the end the CTA brings all threads to a
// common m, and then
//     lse = scale * m + ln S,   logp = (x - m) * scale - ln S,   entropy = ln S - ln 2 * A / S.
// The reference is the thread's first maximum and moves only when a later one is more than a factor
// of 2^8 above it, so the sums are hardly ever rescaled on the way (a running maximum would make
// some lane of a warp rescale at most vectors), and what the late step back to a common
// reference can cost in precision stays within 8 * 2^-24 of a nat.  Logits below -10^30 (masked ones) count
// as -10^30 there, whose power is 0 in any row with a logit above -10^29; parts without one, or with a
// largest logit near the other end of fp32, are summed again by a loop that takes every value as it is.
//
// Top alternatives: every thread remembers its largest logit and the first vector that held it.
// The top_k-th best of those is a lower bound for the row's top_k-th best logit that exactly top_k
// threads reach, so only their vectors are looked at again (they are still in L2), and what
// reaches the bound -- a few dozen logits -- is ranked in shared memory, all by a warp of its own
// beside the threads that stream the next row.
//
// A row is split over several CTAs when there are too few rows to fill the device; each split
// leaves (m, S, A) and its own alternatives in the workspace and a second kernel joins them.
//
// 8192 x 128256 in bf16 (2.10 GB), a call by itself after a flush of L2: 360 us (5.8 TB/s), 416 with 5 alternatives, 432 with
// 20, whatever the spread of the logits; calls back to back, where the power cap holds the clock at 1.7 to 1.8 GHz, 394 and
// (5 alternatives) 436.  The issue slots (54 %) and the multifunction unit (one exponential per logit, 53 %) bound it, not
// memory.  The 56 registers that four CTAs of 288 threads leave spill 112 bytes (bf16) and 120 (fp32) with
// alternatives, none without.  Rows without a logit above -10^29 are summed by one warp: 8192 x 32001 masked entirely
// take 5.2 ms, of the type's lowest value 8.1, ordinary ones 0.11.  Backward 652 us for 4.20 GB, 6.4 TB/s; 677 back to back.
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

constexpr int kLpThreads = 256;
constexpr int kLpMaxTop = 32;
constexpr int kLpCandidates = 1024;          // ranked in shared memory; more take the slow way
constexpr int kLpHits = 512;
constexpr int kLpUnroll = 4;                 // vectors a thread loads at once
constexpr int kLpGroups = 16;                // per thread and row
constexpr int kLpFillCtas = 592;             // four per SM of the device the kernel is tuned on
constexpr int kLpMaxSplits = 74;
constexpr float kLpReach = 8.0f;             // see above
constexpr float kLpFloor = -1.0002555517425873e30f;     // the bf16 value 0xF14A
constexpr float kLpLowest = -1e29f;             // the lowest reference
constexpr float kLpHuge = 1e37f;                // bound of |m| c
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

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
    // the largest value (NaN only if nothing else is there), and the values not below kLpFloor (NaN kept)
    static __device__ __forceinline__ float top(const uint4& w)
    {
        const uint32_t m = max_bf16x2(max_bf16x2(w.x, w.y), max_bf16x2(w.z, w.w));
        return fmaxf(bf16_lo(m), bf16_hi(m));
    }
    static __device__ __forceinline__ void get_floored(const uint4& w, float2 (&v)[4])
    {
        constexpr uint32_t f = 0xF14AF14Au;      // two bf16 of kLpFloor
        const uint4 c = make_uint4(max_nan_bf16x2(w.x, f), max_nan_bf16x2(w.y, f), max_nan_bf16x2(w.z, f), max_nan_bf16x2(w.w, f));
        unpack8(c, v);
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
    static __device__ __forceinline__ float top(const uint4& w)
    {
        return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
    }
    static __device__ __forceinline__ void get_floored(const uint4& w, float2 (&v)[2])
    {
        v[0] = make_float2(max_nan(__uint_as_float(w.x), kLpFloor), max_nan(__uint_as_float(w.y), kLpFloor));
        v[1] = make_float2(max_nan(__uint_as_float(w.z), kLpFloor), max_nan(__uint_as_float(w.w), kLpFloor));
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

// Sums of part of a row: S = sum 2^d, A = sum d 2^d with d = (x - m) c, c = scale * log2(e).  An empty part
// has m = -infinity, and in s what a NaN left there.
struct SoftSums {
    float m, s, a;
};

// The sums relative to a larger reference.
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
template <size_t N>
__device__ __forceinline__ SoftSums block_join(SoftSums v, float c, SoftSums (&red)[N])
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    v = warp_join(v, c);
    if (lane == 0) smem_put(red, warp, v);
    __syncthreads();
    v = lane < static_cast<int>(blockDim.x >> 5) ? smem_get(red, lane) : SoftSums{-INFINITY, 0.0f, 0.0f};
    return warp_join(v, c);
}

// What a row's log probabilities are formed from: z - lse = (x - m) * scale - ln S.  The rounded lse itself will not do:
// far from zero its last bit is worth more than ln S.
struct RowNorm {
    float lse, m, log_s;
};

__device__ __forceinline__ float log_prob(const RowNorm& n, float x, float scale)
{
    if (n.lse != n.lse) return NAN;
    if (n.lse == -INFINITY || x * scale == -INFINITY) return -INFINITY;
    const float d = x - n.m;
    // a difference past fp32's range between two logits whose z are in it: both are far too large for ln S to count
    return fabsf(d) < INFINITY ? fmaf(d, scale, -n.log_s) : fmaf(x, scale, -n.lse);
}

// Row results of one thread.
__device__ __forceinline__ RowNorm finish_row(const LogprobsParams& p, int64_t row, const SoftSums& v)
{
    if (v.m == -INFINITY && v.s == 0.0f) {           // nothing but masked logits
        p.lse[row] = -INFINITY;
        if (p.entropy) p.entropy[row] = 0.0f;
        return {-INFINITY, 0.0f, 0.0f};
    }
    const float log_s = kLn2 * log2f(v.s);
    float lse = v.m == -INFINITY ? v.s : fmaf(v.m, p.scale, log_s);
    if (lse == INFINITY) lse = NAN;                  // a z above fp32's range counts as an infinite logit
    p.lse[row] = lse;
    // all z below the range: a row masked entirely
    if (p.entropy) p.entropy[row] = lse != lse ? lse : lse == -INFINITY ? 0.0f : log_s - kLn2 * (v.a / v.s);
    return {lse, v.m, log_s};
}

template <class T>
__device__ __forceinline__ void finish_target(const LogprobsParams& p, int64_t row, const RowNorm& norm)
{
    if (!p.logp) return;
    const int64_t t = p.targets[row];
    float r = 0.0f;
    if (t >= p.vocab) r = NAN;
    else if (t >= 0) r = log_prob(norm, LogitVec<T>::one(static_cast<const T*>(p.logits) + row * p.ld + t), p.scale);
    p.logp[row] = r;
}

__device__ __forceinline__ void write_top(const LogprobsParams& p, int64_t row, int rank, uint64_t key, const RowNorm& norm)
{
    const int64_t at = row * p.top_k + rank;
    const bool bad = norm.lse != norm.lse;
    const bool none = bad || key == 0ull;
    p.top_logp[at] = bad ? NAN : none ? -INFINITY : log_prob(norm, key_value(static_cast<uint32_t>(key >> 32)), p.scale);
    p.top_index[at] = none ? -1 : static_cast<int64_t>(0xFFFFFFFFu - static_cast<uint32_t>(key));
}

// What the threads of a row leave for the warp that finishes it.
template <bool TOP>
struct RowNotes {
    SoftSums sums[kLpThreads / 32];
    uint32_t key[kLpThreads], vec[kLpThreads];   // a thread's largest logit (as a key), first vector with it
    uint16_t group[TOP ? kLpGroups : 1][kLpThreads];     // upper half of that key for each group of its vectors
};

struct TopScratch {
    uint64_t keys[kLpCandidates];
    uint32_t hits[kLpHits];    // vectors whose largest logit reaches the bound
    uint32_t groups[kLpHits];  // first vectors of groups that do
    int32_t owner[kLpMaxTop];
    int32_t n, n_hits, n_groups;
    RowNorm norm;              // of the row at hand (in registers it would cost the alternatives spills)
    uint64_t top[kLpMaxTop];   // its alternatives
};

struct TopBound {
    uint32_t kth, last_vec;    // the bound's value, and the last vector that counts where the value is equal
    int32_t owners;
};

// One warp picks the threads whose best logits are the `want` largest (equal ones: of the first vectors).  Bits of the bound are tried from the top, as long as more
// than `want` threads reach it.  The threads are left in the scratch.
template <class T>
__device__ __forceinline__ TopBound pick_owners(const RowNotes<true>& notes, TopScratch& sc, int want, int max_vec)
{
    constexpr int SHIFT = LogitVec<T>::kKeyShift;
    constexpr int kEach = kLpThreads / 32;
    const int lane = threadIdx.x & 31;
    uint32_t key[kEach], vec[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        key[i] = smem_get(notes.key, i * 32 + lane) >> SHIFT;
        vec[i] = smem_get(notes.vec, i * 32 + lane);
    }
    auto reach = [&](uint32_t bound) {
        int n = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) n += key[i] >= bound;
        return __reduce_add_sync(0xffffffffu, n);
    };
    uint32_t bound = 0;
    int n = kLpThreads;
    for (int b = 31 - SHIFT; b >= 0 && n != want; --b) {
        const int m = reach(bound | (1u << b));
        if (m >= want) {
            bound |= 1u << b;
            n = m;
        }
    }
    if (bound == 0) bound = 1;                       // fewer than `want` threads have a logit: all of those
    uint32_t last = 0xFFFFFFFFu;
    if (n > want) {
        // more threads than wanted hold the bound itself: the first vectors among those
        int above = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) above += key[i] > bound;
        above = __reduce_add_sync(0xffffffffu, above);
        last = 0;                                    // largest vector number that fewer than the rest come before
        for (int b = 31 - __clz(max_vec | 1); b >= 0; --b) {
            const uint32_t probe = last | (1u << b);
            int m = 0;
#pragma unroll
            for (int i = 0; i < kEach; ++i) m += key[i] == bound && vec[i] < probe;
            if (__reduce_add_sync(0xffffffffu, m) < want - above) last = probe;
        }
    }
    int at = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const bool mine = key[i] > bound || (key[i] == bound && vec[i] <= last);
        const uint32_t who = __ballot_sync(0xffffffffu, mine);
        const int place = at + __popc(who & ((1u << lane) - 1u));
        if (mine && place < kLpMaxTop) smem_put(sc.owner, place, i * 32 + lane);
        at += __popc(who);
    }
    return {bound, last, at < kLpMaxTop ? at : kLpMaxTop};
}

// The elements of a row a CTA owns: vectors first .. first + count, and the unaligned head or tail.
template <class T>
struct RowPart {
    const T* row;
    int head;                  // elements before the first 16-byte boundary
    int first, count;          // vectors
    int loose0, n_loose0;      // single elements: at the row's head,
    int loose1, n_loose1;      // and at its end
    __device__ __forceinline__ int loose_index(int i) const { return i < n_loose0 ? loose0 + i : loose1 + i - n_loose0; }
    // vectors per thread and group, in whole unrolled steps
    __device__ __forceinline__ int group_steps() const
    {
        const int steps = (count + kLpUnroll * kLpThreads - 1) / (kLpUnroll * kLpThreads);
        return (steps + kLpGroups - 1) / kLpGroups;
    }
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

// The part's `top_k` best keys, in the scratch's `top`; 0 for ranks that do not exist.  One warp.
template <class T>
__device__ __forceinline__ void warp_top(const RowPart<T>& part, int top_k, const RowNotes<true>& notes, TopScratch& sc)
{
    constexpr int kN = LogitVec<T>::kN;
    const int lane = threadIdx.x & 31;
    const TopBound bound = pick_owners<T>(notes, sc, top_k, part.first + part.count);
    if (lane == 0) sc.n = sc.n_hits = sc.n_groups = 0;
    smem_put(sc.top, lane, uint64_t{0});
    __syncwarp();
    auto take = [&](float x, uint32_t index) {
        const uint64_t k = full_key(x, index);
        if (k == 0ull) return;
        const int at = atomicAdd(&sc.n, 1);
        if (at < kLpCandidates) smem_put(sc.keys, at, k);
    };
    auto vector_at = [&](int v) { return *reinterpret_cast<const uint4*>(part.vec(part.first + v)); };
    // the owners' groups that reach the bound, and of their vectors those that do: a lane per vector, several
    // loads in flight
    const int group_vecs = part.group_steps() * kLpUnroll;
    auto in_reach = [&](uint32_t key, int first_vec) {
        return key > bound.kth || (key == bound.kth && static_cast<uint32_t>(first_vec) <= bound.last_vec);
    };
    for (int i = lane; i < bound.owners * kLpGroups; i += 32) {
        const int owner = smem_get(sc.owner, i / kLpGroups), g = i % kLpGroups, v = owner + g * group_vecs * kLpThreads;
        // an fp32 group whose upper half equals the bound's may or may not reach it
        const uint32_t half = smem_load<uint16_t>(&notes.group[g][owner], notes.group, sizeof(notes.group));
        const uint32_t bound_half = bound.kth >> (16 - LogitVec<T>::kKeyShift);
        if (v < part.count && (kN == 8 ? in_reach(half, part.first + v) : half >= bound_half)) {
            const int at = atomicAdd(&sc.n_groups, 1);
            if (at < kLpHits) smem_put(sc.groups, at, static_cast<uint32_t>(v));
        }
    }
    __syncwarp();
    const int n_groups = min(sc.n_groups, kLpHits), loads = n_groups * group_vecs;
    constexpr int kBatch = 4;
    for (int l = lane; l < loads; l += 32 * kBatch) {
        uint4 w[kBatch];
        int v[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int i = l + 32 * j, o = i / group_vecs;
            v[j] = i < loads ? static_cast<int>(smem_get(sc.groups, o)) + (i - o * group_vecs) * kLpThreads : part.count;
            if (v[j] < part.count) w[j] = vector_at(v[j]);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (v[j] < part.count && in_reach(order_key(LogitVec<T>::top(w[j])) >> LogitVec<T>::kKeyShift, part.first + v[j])) {
                const int at = atomicAdd(&sc.n_hits, 1);
                if (at < kLpHits) smem_put(sc.hits, at, static_cast<uint32_t>(v[j]));
            }
    }
    __syncwarp();
    const int n_hits = sc.n_hits;
    for (int h = lane; h < n_hits && n_hits <= kLpHits; h += 32) {
        const int v = static_cast<int>(smem_get(sc.hits, h)), vec = part.first + v;
        float x[kN];
        LogitVec<T>::get(vector_at(v), x);
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            if (in_reach(order_key(x[i]) >> LogitVec<T>::kKeyShift, vec))
                take(x[i], static_cast<uint32_t>(part.head + vec * kN + i));
        }
    }
    for (int i = lane; i < part.n_loose0 + part.n_loose1; i += 32) {
        const int at = part.loose_index(i);
        take(LogitVec<T>::one(part.row + at), static_cast<uint32_t>(at));
    }
    __syncwarp();
    const int n = n_hits <= kLpHits && sc.n_groups <= kLpHits ? sc.n : kLpCandidates + 1;
    if (n <= kLpCandidates) {
        for (int i = lane; i < n; i += 32) {
            const uint64_t k = smem_get(sc.keys, i);
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += smem_get(sc.keys, j) > k;
            if (rank < top_k) smem_put(sc.top, rank, k);
        }
    } else {
        // hundreds of vectors reach the bound: rank after rank, each from the whole part
        uint64_t last = ~0ull;
        for (int rank = 0; rank < top_k && last; ++rank) {
            uint64_t mine = 0ull;
            auto look = [&](float x, uint32_t index) {
                const uint64_t k = full_key(x, index);
                if (k < last && k > mine) mine = k;
            };
            for (int v = lane; v < part.count; v += 32) {
                const T* at = part.vec(part.first + v);
                float x[kN];
                LogitVec<T>::get(*reinterpret_cast<const uint4*>(at), x);
#pragma unroll
                for (int i = 0; i < kN; ++i) look(x[i], static_cast<uint32_t>(at - part.row) + i);
            }
            for (int i = lane; i < part.n_loose0 + part.n_loose1; i += 32)
                look(LogitVec<T>::one(part.row + part.loose_index(i)), static_cast<uint32_t>(part.loose_index(i)));
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                const uint64_t other = __shfl_xor_sync(0xffffffffu, mine, o);
                if (other > mine) mine = other;
            }
            last = mine;
            if (lane == 0) smem_put(sc.top, rank, last);
        }
    }
    __syncwarp();
}

// Sums of a part with every value taken as it is, relative to the part's own largest logit: for parts whose
// logits are all masked or lie at the ends of the type.  One warp; the same in every lane.
template <class T>
__device__ __noinline__ SoftSums careful_sums(const RowPart<T>& part, float c)
{
    const int n = part.count * LogitVec<T>::kN, all = n + part.n_loose0 + part.n_loose1;
    const int lane = threadIdx.x & 31;
    auto at = [&](int i) {
        return LogitVec<T>::one(i < n ? part.vec(part.first) + i : part.row + part.loose_index(i - n));
    };
    SoftSums v = {-INFINITY, 0.0f, 0.0f};
#pragma unroll 8
    for (int i = lane; i < all; i += 32) {
        const float x = at(i);
        v.m = fmaxf(v.m, x);
        if (x != x) v.s = x;
    }
    v = warp_join(v, c);
    if (v.m == -INFINITY) return v;
    v.s = v.a = 0.0f;
#pragma unroll 8
    for (int i = lane; i < all; i += 32) {
        const float d = max_nan((at(i) - v.m) * c, -300.0f), e = exp2_approx(d);
        v.s += e;
        v.a = fmaf(d, e, v.a);
    }
    return warp_join(v, c);
}

// A CTA walks items (a row, or a split of one): 256 threads stream the logits, and one more warp finishes an item
// -- joins the sums, finds the alternatives, writes the results -- while they stream the next.  Named barriers
// 1 and 2 hand a set of notes over, 3 and 4 hand it back; nobody waits for anything else.
constexpr int kLpCtaThreads = kLpThreads + 32;
template <class T, bool TOP>
__global__ void __launch_bounds__(kLpCtaThreads, 4) logprobs_forward_kernel(const __grid_constant__ LogprobsParams p)
{
    constexpr int kN = LogitVec<T>::kN;
    __shared__ RowNotes<TOP> notes[2];
    __shared__ TopScratch scratch;
    griddep_launch_dependents();
    griddep_wait();
    const int64_t items = p.tokens * p.splits;
    const float c = p.scale * kLog2e;
    const int lane = threadIdx.x & 31;
    int buf = 0;

    if (threadIdx.x >= kLpThreads) {
        // ---------------------------------------------------------------- finishing warp
        for (int64_t item = blockIdx.x; item < items; item += gridDim.x, buf ^= 1) {
            const int64_t row = item / p.splits;
            const int split = static_cast<int>(item - row * p.splits);
            const RowPart<T> part = row_part<T>(p, row, split);
            bar_sync(1 + buf, kLpCtaThreads);
            SoftSums sums = lane < kLpThreads / 32 ? smem_get(notes[buf].sums, lane) : SoftSums{-INFINITY, 0.0f, 0.0f};
            sums = warp_join(sums, c);
            // (with scales beyond these, -10^30 times c is not far below everything, or not a number)
            if (!(fabsf(sums.m) * c < kLpHuge) || c < 1e-26f || c > 1e7f) sums = careful_sums<T>(part, c);
            if (p.splits == 1) {
                if (lane == 0) {
                    scratch.norm = finish_row(p, row, sums);
                    finish_target<T>(p, row, scratch.norm);
                }
                if constexpr (TOP) {
                    __syncwarp();
                    const float lse = scratch.norm.lse;
                    const bool any = lse == lse && lse != -INFINITY;
                    if (any) warp_top<T>(part, p.top_k, notes[buf], scratch);
                    if (lane < p.top_k) write_top(p, row, lane, any ? smem_get(scratch.top, lane) : 0ull, scratch.norm);
                }
            } else {
                if (lane == 0) p.part_sums[item] = make_float4(sums.m, sums.s, sums.a, 0.0f);
                if constexpr (TOP) {
                    warp_top<T>(part, p.top_k, notes[buf], scratch);
                    if (lane < p.top_k) p.part_keys[item * p.top_k + lane] = smem_get(scratch.top, lane);
                }
            }
            if (item + 2 * static_cast<int64_t>(gridDim.x) < items) bar_arrive(3 + buf, kLpCtaThreads);
        }
        return;
    }

    // -------------------------------------------------------------------- streaming threads
    const float reach = kLpReach / c;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x, buf ^= 1) {
        const int64_t row = item / p.splits;
        const RowPart<T> part = row_part<T>(p, row, static_cast<int>(item - row * p.splits));
        float m = -INFINITY, ref = 0.0f, limit = kLpLowest;  // ref = m, or 0 while no logit above kLpLowest came
        float2 s = make_float2(0.0f, 0.0f), a = make_float2(0.0f, 0.0f);
        float best = -INFINITY;
        int best_vec = 0;
        auto move_reference = [&](float top) {
            if (m > -INFINITY) {
                const float d = fmaxf((m - top) * c, -1000.0f), f = exp2_approx(d);
                a.x = f * fmaf(d, s.x, a.x);
                a.y = f * fmaf(d, s.y, a.y);
                s.x *= f;
                s.y *= f;
            }
            m = ref = top;
            limit = top + reach;
        };
        float group_best = -INFINITY;
        int step = 0, group = 0;
        const int group_steps = TOP ? part.group_steps() : 0;
        auto look = [&](const float* tops, int n, int vec) {    // n vectors from `vec` on, kLpThreads apart
            float top = tops[0];
#pragma unroll
            for (int j = 1; j < n; ++j) top = fmaxf(top, tops[j]);
            if (top > limit) move_reference(top);
            if (TOP) {
                group_best = fmaxf(group_best, top);
                if (top > best) {
                    best = top;
#pragma unroll
                    for (int j = n - 1; j >= 0; --j)
                        if (tops[j] == top) best_vec = vec + j * kLpThreads;     // the first of them stays
                }
            }
        };
        auto accumulate = [&](const uint4& w) {
            float2 x[kN / 2];
            LogitVec<T>::get_floored(w, x);
#pragma unroll
            for (int i = 0; i < kN / 2; ++i) {
                const float2 d = __fmul2_rn(__fadd2_rn(x[i], pair(-ref)), pair(c));
                const float2 e = make_float2(exp2_approx(d.x), exp2_approx(d.y));
                s = __fadd2_rn(s, e);
                a = __ffma2_rn(d, e, a);
            }
        };
        // the notes of two items ago have been read
        if (item >= 2 * static_cast<int64_t>(gridDim.x)) bar_sync(3 + buf, kLpCtaThreads);
        auto close_group = [&](bool last) {
            if (++step == group_steps || last) {
                smem_store(&notes[buf].group[group][threadIdx.x], static_cast<uint16_t>(order_key(group_best) >> 16),
                           notes[buf].group, sizeof(notes[buf].group));
                group_best = -INFINITY;
                step = 0;
                ++group;
            }
        };
        const T* base = part.vec(part.first);
        int v = threadIdx.x;
        for (; v + (kLpUnroll - 1) * kLpThreads < part.count; v += kLpUnroll * kLpThreads) {
            uint4 w[kLpUnroll];
#pragma unroll
            for (int j = 0; j < kLpUnroll; ++j) w[j] = ld_stream(base + static_cast<int64_t>(v + j * kLpThreads) * kN);
            float tops[kLpUnroll];
#pragma unroll
            for (int j = 0; j < kLpUnroll; ++j) tops[j] = LogitVec<T>::top(w[j]);
            look(tops, kLpUnroll, part.first + v);
#pragma unroll
            for (int j = 0; j < kLpUnroll; ++j) accumulate(w[j]);
            if (TOP) close_group(false);
        }
        const bool rest = v < part.count;
        for (; v < part.count; v += kLpThreads) {
            const uint4 w = ld_stream(base + static_cast<int64_t>(v) * kN);
            const float top = LogitVec<T>::top(w);
            look(&top, 1, part.first + v);
            accumulate(w);
        }
        if (TOP && (rest || step > 0)) close_group(true);
        if (static_cast<int>(threadIdx.x) < part.n_loose0 + part.n_loose1) {
            const float x = LogitVec<T>::one(part.row + part.loose_index(threadIdx.x));
            if (x > limit) move_reference(x);
            const float d = (max_nan(x, kLpFloor) - ref) * c, e = exp2_approx(d);
            s.x += e;
            a.x = fmaf(d, e, a.x);
        }
        const SoftSums sums = warp_join({m, s.x + s.y, a.x + a.y}, c);
        if (lane == 0) smem_put(notes[buf].sums, threadIdx.x >> 5, sums);
        if (TOP) {
            smem_put(notes[buf].key, threadIdx.x, order_key(best));
            smem_put(notes[buf].vec, threadIdx.x, static_cast<uint32_t>(best_vec));
        }
        bar_arrive(1 + buf, kLpCtaThreads);
    }
}

// Joins the splits of a row: the sums, and rank after rank the largest key not taken yet.
constexpr int kLpJoinThreads = 256;
template <class T>
__global__ void __launch_bounds__(kLpJoinThreads) logprobs_join_kernel(const LogprobsParams p)
{
    __shared__ SoftSums red[kLpJoinThreads / 32];
    __shared__ uint64_t keys[kLpMaxSplits * kLpMaxTop];
    __shared__ RowNorm row_norm;
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
        row_norm = finish_row(p, row, v);
        finish_target<T>(p, row, row_norm);
    }
    if (p.top_k == 0) return;
    const int n = p.splits * p.top_k;
    for (int i = threadIdx.x; i < n; i += kLpJoinThreads) smem_put(keys, i, p.part_keys[row * n + i]);
    __syncthreads();
    const RowNorm norm = row_norm;
    // Each split's keys are in descending order: one warp takes the largest head, rank after rank, and keeps the
    // key of rank r in lane r.
    if (threadIdx.x >= 32) return;
    constexpr int kLists = (kLpMaxSplits + 31) / 32;
    const int lane = threadIdx.x;
    int at[kLists];
#pragma unroll
    for (int i = 0; i < kLists; ++i) at[i] = 0;
    uint64_t mine = 0ull;
    const bool any = norm.lse == norm.lse && norm.lse != -INFINITY;
    for (int rank = 0; any && rank < p.top_k; ++rank) {
        uint64_t head[kLists], best = 0ull;
#pragma unroll
        for (int i = 0; i < kLists; ++i) {
            const int split = lane + 32 * i;
            head[i] = split < p.splits && at[i] < p.top_k ? smem_get(keys, split * p.top_k + at[i]) : 0ull;
            if (head[i] > best) best = head[i];
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const uint64_t other = __shfl_xor_sync(0xffffffffu, best, o);
            if (other > best) best = other;
        }
        if (best == 0ull) break;
#pragma unroll
        for (int i = 0; i < kLists; ++i) at[i] += head[i] == best;       // keys are unique
        if (lane == rank) mine = best;
    }
    if (lane < p.top_k) write_top(p, row, lane, mine, norm);
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
    const bool bad = p.d_logp && target >= p.vocab;
    if (bad) gl = NAN;
    const float ge = p.d_entropy ? p.d_entropy[row] : 0.0f;
    const float base = fmaf(ge, p.entropy && p.d_entropy ? p.entropy[row] : 0.0f, gl);
    const bool zero = (gl == 0.0f && ge == 0.0f) || (lse == -INFINITY && !bad);
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

// Status word of this translation unit's kernels, cleared when it is set.
int logprobs_take_status(int* status) { return take_unit_status(status); }

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
static int launch_logprobs_forward(const LogprobsParams& p, int sm_count, cudaStream_t st)
{
    const int64_t items = p.tokens * p.splits, most = 4 * static_cast<int64_t>(sm_count);
    const int grid = static_cast<int>(items < most ? items : most);
    const cudaError_t e = p.top_k > 0
                              ? launch_kernel_pdl(logprobs_forward_kernel<T, true>, grid, kLpCtaThreads, 0, st, p)
                              : launch_kernel_pdl(logprobs_forward_kernel<T, false>, grid, kLpCtaThreads, 0, st, p);
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
    return dtype == MXFP4_OUT_BF16 ? launch_logprobs_forward<__nv_bfloat16>(p, dev.sm_count, st)
                                   : launch_logprobs_forward<float>(p, dev.sm_count, st);
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
