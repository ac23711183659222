// Token embeddings: scaled lookup, and the gradient of the table (see include/mxfp4.h).
//
// Backward.  The positions are sorted by their ids, positions of the same id in their order, and the first of each id's
// run is noted (a note counts only where the sorted ids confirm it, so the notes need no clearing).  Then
//   - the sorted positions are shared out evenly, and gradients of equal ids are added in fp32 in the order of their
//     positions; where a run spans shares, its partial sums are joined in the order of the shares;
//   - beside that the rows without tokens of a dense gradient are set to zero.  Small CTAs in the device's own order keep
//     the rows being written close together: 128256 rows of 16 KB take 273 us that way (7.3 TB/s), 338 from CTAs that stay
//     and take rows in turn.
// 16384 tokens of 4096 columns, fp32 gradient of 128256 rows: 344 us for 2.24 GB, as fast as a copy (19 us of it the sort;
// 360 with the sums before the zeros, 378 with sums from registers, 464 with zeros first); 777 tokens of 2048, bf16, 32001
// rows: 30 us for 134 MB.
// No floating-point atomics: results depend on the inputs alone.
//
// Up to 4096 positions are sorted by counting, for each, the smaller ones: 2 T^2 comparisons over the whole device, one
// launch without any exchange.  Longer texts take a radix sort by a cluster of eight CTAs, 9 bits per pass from the lowest:
// each CTA counts the digits of its eighth of the positions, reads the other CTAs' counts through distributed shared
// memory and places its positions, 4096 at a time, behind the smaller digits, the earlier CTAs' and its own earlier ones.
// Ids without a row sort behind all others.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/mxfp4.h"
#include "host_common.cuh"
#include "ptx_sm100.cuh"
#include "row_io.cuh"
#include "tma_host.cuh"

namespace mxfp4 {

__device__ __forceinline__ void load8_stream(const __nv_bfloat16* p, float2 (&v)[4]) { unpack8(ld_stream(p), v); }

__device__ __forceinline__ void load8_stream(const float* p, float2 (&v)[4])
{
    const uint4 a = ld_stream(p), b = ld_stream(p + 4);
    v[0] = make_float2(__uint_as_float(a.x), __uint_as_float(a.y));
    v[1] = make_float2(__uint_as_float(a.z), __uint_as_float(a.w));
    v[2] = make_float2(__uint_as_float(b.x), __uint_as_float(b.y));
    v[3] = make_float2(__uint_as_float(b.z), __uint_as_float(b.w));
}

// ------------------------------------------------------------------ lookup
struct LookupParams {
    const int64_t* ids;
    const void* table;
    void* out;
    int64_t ld_table, ld_out, vocab;
    int64_t items;               // tokens * width / 8
    int32_t per_row;             // width / 8
    float scale;
};

constexpr int kLookupThreads = 256;
constexpr int kLookupUnroll = 4; // rows' pieces in flight per thread

template <class In, class Out>
__global__ void __launch_bounds__(kLookupThreads) lookup_kernel(const LookupParams p)
{
    griddep_launch_dependents();
    griddep_wait();
    const int64_t first = static_cast<int64_t>(blockIdx.x) * (kLookupThreads * kLookupUnroll) + threadIdx.x;
    float2 v[kLookupUnroll][4];
    int64_t row[kLookupUnroll], col[kLookupUnroll], id[kLookupUnroll];
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) {
        const int64_t i = first + u * kLookupThreads;
        row[u] = i / p.per_row;
        col[u] = (i - row[u] * p.per_row) * 8;
        id[u] = i < p.items ? __ldg(p.ids + row[u]) : -1;
    }
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) {
        if (id[u] >= 0 && id[u] < p.vocab) {
            load8_stream(static_cast<const In*>(p.table) + id[u] * p.ld_table + col[u], v[u]);
        } else {
            const float none = id[u] < 0 ? 0.0f : NAN;
            for (int j = 0; j < 4; ++j) v[u][j] = make_float2(none, none);
        }
    }
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) {
        if (first + u * kLookupThreads >= p.items) break;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[u][j] = id[u] < 0 ? v[u][j] : make_float2(v[u][j].x * p.scale, v[u][j].y * p.scale);
        store8(static_cast<Out*>(p.out) + row[u] * p.ld_out + col[u], v[u]);
    }
}

// ------------------------------------------------------------------ sort
struct SortParams {
    const int64_t* ids;
    uint2* a;                    // (id, position), in turn source and destination; the result is in a
    uint2* b;
    uint32_t* first;             // [vocab]: where the id's run begins
    int32_t tokens;
    int32_t passes;
    int64_t vocab;
};

__device__ __forceinline__ uint32_t sort_key(const SortParams& p, int64_t id)
{
    return static_cast<uint32_t>(id < 0 || id >= p.vocab ? p.vocab : id);
}

constexpr int kRankMost = 4096;                    // positions
constexpr int kRankWarps = 8;

// 32 positions per CTA, one per lane; every warp compares them with an eighth of all.
__global__ void __launch_bounds__(kRankWarps * 32) rank_kernel(const __grid_constant__ SortParams p)
{
    __shared__ uint4 keys[kRankMost / 4];
    __shared__ uint32_t less[kRankWarps][32], same[kRankWarps][32];
    griddep_launch_dependents();
    griddep_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int quads = (p.tokens + 3) / 4;
    for (int i = threadIdx.x; i < quads; i += kRankWarps * 32) {
        uint32_t k[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) k[j] = 4 * i + j < p.tokens ? sort_key(p, p.ids[4 * i + j]) : 0xFFFFFFFFu;
        smem_put(keys, i, make_uint4(k[0], k[1], k[2], k[3]));
    }
    __syncthreads();
    const int mine = blockIdx.x * 32 + lane;
    const uint32_t key = mine < p.tokens ? sort_key(p, p.ids[mine]) : 0u;
    const int share = (quads + kRankWarps - 1) / kRankWarps;
    const int begin = warp * share, end = min(quads, begin + share);
    uint32_t n_less = 0, n_same = 0;               // smaller ids; equal ones at earlier positions
#pragma unroll 4
    for (int i = begin; i < end; ++i) {
        const uint4 k = smem_get(keys, i);
        n_less += (k.x < key) + (k.y < key) + (k.z < key) + (k.w < key);
        n_same += (k.x == key && 4 * i < mine) + (k.y == key && 4 * i + 1 < mine) + (k.z == key && 4 * i + 2 < mine) +
                  (k.w == key && 4 * i + 3 < mine);
    }
    smem_store(&less[warp][lane], n_less, less, sizeof(less));
    smem_store(&same[warp][lane], n_same, same, sizeof(same));
    __syncthreads();
    if (warp != 0 || mine >= p.tokens) return;
    n_less = n_same = 0;
    for (int w = 0; w < kRankWarps; ++w) {
        n_less += smem_load<uint32_t>(&less[w][lane], less, sizeof(less));
        n_same += smem_load<uint32_t>(&same[w][lane], same, sizeof(same));
    }
    p.a[n_less + n_same] = make_uint2(key, static_cast<uint32_t>(mine));
    if (n_same == 0 && key < p.vocab) p.first[key] = n_less;
}

constexpr int kSortCtas = 8;                       // one cluster
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortItems = 4;                      // positions per thread and round
constexpr int kSortBits = 9;
constexpr int kSortBins = 1 << kSortBits;

struct SortSmem {
    uint32_t counts[kSortBins];                    // of this CTA's positions
    uint32_t start[kSortBins];                     // where the next position with this digit goes
    uint32_t warp_counts[kSortWarps][kSortBins];   // digits of a round, then where each warp's start
    uint32_t sums[kSortWarps];
};

__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t cluster_addr)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_addr) : "memory");
    return v;
}

__global__ void __cluster_dims__(kSortCtas, 1, 1) __launch_bounds__(kSortThreads, 1) sort_kernel(const __grid_constant__ SortParams p)
{
    extern __shared__ uint8_t smem_raw[];
    SortSmem& s = *reinterpret_cast<SortSmem*>(smem_align_1024(smem_raw));
    griddep_launch_dependents();
    griddep_wait();
    const uint32_t rank = cluster_ctarank();
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    const int share = (p.tokens + kSortCtas - 1) / kSortCtas;
    const int begin = min(p.tokens, static_cast<int>(rank) * share), end = min(p.tokens, begin + share);
    const uint2* from = nullptr;
    for (int pass = 0; pass < p.passes; ++pass) {
        uint2* to = (p.passes - pass) & 1 ? p.a : p.b;
        const int shift = pass * kSortBits;
        auto entry = [&](int i) {
            if (from) return from[i];
            return make_uint2(sort_key(p, p.ids[i]), static_cast<uint32_t>(i));
        };
        auto digit_of = [&](const uint2& e) { return static_cast<int>((e.x >> shift) & (kSortBins - 1)); };
        if (t < kSortBins) smem_put(s.counts, t, 0u);
        __syncthreads();
        for (int i = begin + t; i < end; i += kSortThreads) {
            const int d = digit_of(entry(i));
            if (smem_within(s.counts, d)) atomicAdd(s.counts + d, 1u);
        }
        cluster_sync_all();
        // positions of smaller digits, and of this digit in earlier CTAs
        uint32_t all = 0, before = 0;
        if (t < kSortBins && smem_within(s.counts, t)) {
            const uint32_t mine = smem_u32(s.counts + t);
            for (uint32_t c = 0; c < kSortCtas; ++c) {
                const uint32_t n = ld_cluster_u32(map_to_cta(mine, c));
                all += n;
                if (c < rank) before += n;
            }
        }
        uint32_t upto = all;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += v;
        }
        if (lane == 31) smem_put(s.sums, warp, upto);
        __syncthreads();
        if (t < kSortBins) {
            uint32_t base = 0;
            for (int w = 0; w < warp; ++w) base += smem_get(s.sums, w);
            smem_put(s.start, t, base + upto - all + before);
        }
        // a round of positions: 128 consecutive ones per warp, four per lane
        constexpr int kRound = kSortThreads * kSortItems;
        uint2 e[kSortItems];
        auto load = [&](int i0) {
#pragma unroll
            for (int j = 0; j < kSortItems; ++j) {
                const int i = i0 + (warp * kSortItems + j) * 32 + lane;
                e[j] = i < end ? entry(i) : make_uint2(0u, 0u);
            }
        };
        load(begin);
        for (int i0 = begin; i0 < end; i0 += kRound) {
            for (int i = t; i < kSortWarps * kSortBins; i += kSortThreads) smem_store(&s.warp_counts[0][0] + i, 0u, s.warp_counts, sizeof(s.warp_counts));
            __syncthreads();
            int at_digit[kSortItems];
#pragma unroll
            for (int j = 0; j < kSortItems; ++j) {
                const bool in = i0 + (warp * kSortItems + j) * 32 + lane < end;
                const int d = digit_of(e[j]);
                // lanes with the same digit (those past the end among themselves)
                const uint32_t same = __match_any_sync(0xffffffffu, in ? d : kSortBins + lane);
                const int ahead = __popc(same & ((1u << lane) - 1));
                uint32_t* count = &s.warp_counts[warp][d];
                const uint32_t n = smem_load<uint32_t>(count, s.warp_counts, sizeof(s.warp_counts));
                __syncwarp();
                if (in && ahead == 0) smem_store(count, n + __popc(same), s.warp_counts, sizeof(s.warp_counts));
                __syncwarp();
                at_digit[j] = in ? static_cast<int>(n) + ahead : -1;
            }
            __syncthreads();
            if (t < kSortBins) {
                uint32_t at = smem_get(s.start, t);
#pragma unroll 8
                for (int w = 0; w < kSortWarps; ++w) {
                    uint32_t* c = &s.warp_counts[w][t];
                    const uint32_t n = smem_load<uint32_t>(c, s.warp_counts, sizeof(s.warp_counts));
                    smem_store(c, at, s.warp_counts, sizeof(s.warp_counts));
                    at += n;
                }
                smem_put(s.start, t, at);
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kSortItems; ++j) {
                const uint32_t at = smem_load<uint32_t>(&s.warp_counts[warp][digit_of(e[j])], s.warp_counts, sizeof(s.warp_counts)) + at_digit[j];
                if (at_digit[j] >= 0 && at < static_cast<uint32_t>(p.tokens)) to[at] = e[j];
            }
            load(i0 + kRound);
            __syncthreads();
        }
        cluster_sync_all();      // everything is placed, and the counts have been read
        from = to;
    }
    for (int i = begin + t; i < end; i += kSortThreads) {
        const uint32_t id = p.a[i].x;
        if (id < p.vocab && (i == 0 || p.a[i - 1].x != id)) p.first[id] = static_cast<uint32_t>(i);
    }
}

// ------------------------------------------------------------------ sums
struct SumParams {
    const uint2* sorted;         // (id, position)
    const void* grads;
    void* table;
    float* parts;                // [share][goes on, begins][width]
    int64_t ld_grads, ld_table;
    int32_t tokens, width;
    int32_t share;               // sorted positions per warp
    int32_t shares;
    uint32_t vocab;
    int32_t slabs;               // pieces of kSlab columns
    int32_t accumulate;
    float scale;
};

constexpr int kSumWarps = 8;
constexpr int kSumAll = 148 * kSumWarps;           // shares times slabs; a constant, so that results do not depend on the device
constexpr int kSlab = 1024;                        // columns of a warp, 32 per lane
constexpr int kRingBytes = 24576;                  // per warp
constexpr int kLeastShare = 8;

struct SumSmem {
    alignas(128) uint8_t ring[kSumWarps][kRingBytes];
    uint64_t full[kSumWarps][kRingBytes / (kSlab * 2)];
    int abort_flag;
};

// 8 columns each of four groups of 256 per lane
struct RowSum {
    float2 v[4][4];

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[g][j] = make_float2(0.0f, 0.0f);
    }
    __device__ __forceinline__ void add(int g, const float2 (&w)[4])
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[g][j] = make_float2(v[g][j].x + w[j].x, v[g][j].y + w[j].y);
    }
};

// Eight columns of a row from their sums.
template <class Out>
__device__ __forceinline__ void write8(const SumParams& p, uint32_t id, int col, float2 (&sum)[4])
{
    Out* to = static_cast<Out*>(p.table) + id * p.ld_table + col;
    float2 old[4] = {};
    if (p.accumulate) load8_stream(to, old);
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] = make_float2(fmaf(sum[j].x, p.scale, old[j].x), fmaf(sum[j].y, p.scale, old[j].y));
    store8(to, sum);
}

template <class Out>
__device__ __forceinline__ void write_row(const SumParams& p, uint32_t id, int col, RowSum& s)
{
#pragma unroll
    for (int g = 0; g < 4; ++g)
        if (col + g * 256 < p.width) write8<Out>(p, id, col + g * 256, s.v[g]);
}

// A warp per share of the sorted positions and 1024 columns.  The rows come through a ring of bulk copies in shared memory,
// 24 KB per warp, whatever runs they belong to: most runs are one position long, and what a warp could keep on its way
// in registers is one or two rows.  The part of a run that began in an earlier share is partial sum 0 of this share, the
// part of one that goes on behind it partial sum 1.
template <class In, class Out>
__global__ void __launch_bounds__(kSumWarps * 32, 1) sum_kernel(const __grid_constant__ SumParams p)
{
    extern __shared__ uint8_t smem_raw[];
    SumSmem& sm = *reinterpret_cast<SumSmem*>(smem_align_1024(smem_raw));
    constexpr int kRowBytes = kSlab * sizeof(In), kSlots = kRingBytes / kRowBytes;
    const int warp = threadIdx.x >> 5, lane = lane_id();
    if (threadIdx.x == 0) {
        sm.abort_flag = 0;
        for (int w = 0; w < kSumWarps; ++w)
            for (int i = 0; i < kSlots; ++i) mbar_init(&sm.full[w][i], 1);
        fence_barrier_init();
    }
    __syncthreads();
    griddep_wait();
    griddep_launch_dependents();                   // not before the wait: see fill_join_kernel
    uint8_t* ring = sm.ring[warp];
    uint64_t* full = sm.full[warp];
    int slot = 0;                                  // of the row to be added next
    uint32_t parity = 0;
    // neighbouring units go to different SMs
    for (int u = blockIdx.x + gridDim.x * warp; u < p.shares * p.slabs; u += gridDim.x * kSumWarps) {
        const int share = u / p.slabs, col0 = (u - share * p.slabs) * kSlab, col = col0 + lane * 8;
        const int begin = share * p.share, end = min(p.tokens, begin + p.share);
        const uint32_t bytes = static_cast<uint32_t>(min(kSlab, p.width - col0)) * sizeof(In);
        const In* grads = static_cast<const In*>(p.grads) + col0;
        const uint32_t before = begin > 0 ? p.sorted[begin - 1].x : 0xFFFFFFFFu;
        const uint32_t after = end < p.tokens ? p.sorted[end].x : 0xFFFFFFFFu;
        // 64 positions' entries from `base` on
        auto entries = [&](int i) { return i < end ? p.sorted[i] : make_uint2(0xFFFFFFFFu, 0u); };
        int base = begin;
        uint2 near = entries(begin + lane), far = entries(begin + 32 + lane);
        auto id_of = [&](int i) { return __shfl_sync(0xffffffffu, i - base < 32 ? near.x : far.x, (i - base) & 31); };
        auto issue = [&](int i, int to) {
            const uint32_t pos = __shfl_sync(0xffffffffu, i - base < 32 ? near.y : far.y, (i - base) & 31);
            if (id_of(i) < p.vocab && lane == 0) {
                mbar_arrive_expect_tx(&full[to], bytes);
                bulk_load_1d(ring + to * kRowBytes, grads + pos * p.ld_grads, bytes, &full[to]);
            }
        };
        for (int i = 0; i < kSlots; ++i) issue(begin + i, slot + i < kSlots ? slot + i : slot + i - kSlots);
        RowSum s;
        s.clear();
        uint32_t id = id_of(begin);
        bool first = true, alive = true;           // `id` is the share's first
        auto finish = [&](bool last) {
            const int part = first && id == before ? 0 : last && id == after ? 1 : -1;
            if (part < 0) {
                write_row<Out>(p, id, col, s);
                return;
            }
            float* to = p.parts + (static_cast<int64_t>(share) * 2 + part) * p.width + col;
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if (col + g * 256 < p.width) store8(to + g * 256, s.v[g]);
        };
        int i = begin;
        for (; i < end; ++i) {
            const uint32_t next = id_of(i);
            if (next >= p.vocab) break;            // these come last
            if (next != id) {
                finish(false);
                s.clear();
                id = next;
                first = false;
            }
            if (!mbar_wait(&full[slot], parity, &sm.abort_flag)) {
                alive = false;
                break;
            }
            const uint8_t* row = ring + slot * kRowBytes;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float2 v[4];
                if constexpr (sizeof(In) == 2) {
                    unpack8(smem_load<uint4>(row + g * 512 + lane * 16, ring, kRingBytes), v);
                } else {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const float4 f = smem_load<float4>(row + g * 1024 + lane * 32 + k * 16, ring, kRingBytes);
                        v[2 * k] = make_float2(f.x, f.y);
                        v[2 * k + 1] = make_float2(f.z, f.w);
                    }
                }
                s.add(g, v);
            }
            __syncwarp();
            if (i + 1 - base == 32) {
                base += 32;
                near = far;
                far = entries(base + 32 + lane);
            }
            issue(i + kSlots, slot);
            if (++slot == kSlots) {
                slot = 0;
                parity ^= 1;
            }
        }
        if (!alive) {                              // given up: what is in flight lands before the CTA leaves
            linger();
            break;
        }
        if (i > begin) finish(i == end);
    }
}

// The rows without tokens of a dense gradient, eight per CTA, and after them the rows whose runs span shares: a warp per share
// that one begins in and 256 columns.
//
// The zeros are written beside the sums before them in the stream: other rows, and a CTA of this kernel starts only after
// every CTA of that one has seen all work before it complete.  What this kernel reads of it comes past L1.  Every CTA waits
// for the sums before it ends, so that what follows in the stream comes after both.
struct FillParams {
    const uint32_t* first;
    int64_t pitch;               // bytes
    int32_t vectors;             // 16-byte pieces per row
    int32_t blocks;              // of zeros
    int32_t slabs;               // pieces of 256 columns
};

constexpr int kFillRows = 8;

template <class Out>
__global__ void __launch_bounds__(kFillRows * 32) fill_join_kernel(const __grid_constant__ SumParams p, const __grid_constant__ FillParams f)
{
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31;
    if (static_cast<int>(blockIdx.x) < f.blocks) {
        const uint32_t row = blockIdx.x * kFillRows + (threadIdx.x >> 5);
        if (row < p.vocab) {
            const uint32_t at = __ldcg(f.first + row);
            const bool any = at < static_cast<uint32_t>(p.tokens) && __ldcg(&p.sorted[at].x) == row &&
                             (at == 0 || __ldcg(&p.sorted[at - 1].x) != row);
            uint8_t* to = static_cast<uint8_t*>(p.table) + row * f.pitch;
            for (int i = lane; i < f.vectors && !any; i += 32) st_stream(to + i * 16, make_uint4(0u, 0u, 0u, 0u));
        }
        griddep_wait();
        return;
    }
    griddep_wait();
    const int64_t u = static_cast<int64_t>(blockIdx.x - f.blocks) * kFillRows + (threadIdx.x >> 5);
    const int share = static_cast<int>(u / f.slabs), col = (static_cast<int>(u - static_cast<int64_t>(share) * f.slabs) * 32 + lane) * 8;
    if (share + 1 >= p.shares) return;
    const int begin = share * p.share;
    const uint32_t id = __ldcg(&p.sorted[begin + p.share].x);
    // it goes on in the next share, and begins in this one
    if (id >= p.vocab || __ldcg(&p.sorted[begin + p.share - 1].x) != id || (begin > 0 && __ldcg(&p.sorted[begin - 1].x) == id)) return;
    const float* parts = p.parts + static_cast<int64_t>(share) * 2 * p.width + min(col, p.width - 8);
    float2 sum[4];
    load8_stream(parts + p.width, sum);
    for (int c = share + 1;; c += 32) {
        const bool in = c + lane < p.shares && __ldcg(&p.sorted[(c + lane) * p.share].x) == id;
        const uint32_t out = ~__ballot_sync(0xffffffffu, in);
        const int n = out == 0 ? 32 : __ffs(out) - 1;
        parts = p.parts + static_cast<int64_t>(c) * 2 * p.width + min(col, p.width - 8);
#pragma unroll 4
        for (int k = 0; k < n; ++k) {
            float2 v[4];
            load8_stream(parts + static_cast<int64_t>(k) * 2 * p.width, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] = make_float2(sum[j].x + v[j].x, sum[j].y + v[j].y);
        }
        if (n < 32) break;
    }
    if (col < p.width) write8<Out>(p, id, col, sum);
}

template <class In, class Out>
static int launch_sums(const SumParams& s, int64_t units, int sm_count, cudaStream_t st)
{
    static PerDeviceOnce once;
    const size_t smem = sizeof(SumSmem) + 1024;
    const int rc = ensure_smem_attribute(once, sum_kernel<In, Out>, smem);
    if (rc != MXFP4_OK) return rc;
    const int grid = static_cast<int>(std::min<int64_t>(units, sm_count));
    return launch_kernel_pdl(sum_kernel<In, Out>, grid, kSumWarps * 32, smem, st, s) == cudaSuccess ? MXFP4_OK : MXFP4_ERR_CUDA;
}

static int64_t sum_slabs(int64_t width) { return (width + kSlab - 1) / kSlab; }

// Sorted positions per warp: all warps of the device have one share of one slab, none less than a few positions.
static int64_t sum_share(int64_t tokens, int64_t width)
{
    const int64_t slabs = sum_slabs(width), shares = slabs < kSumAll ? kSumAll / slabs : 1;
    return std::max<int64_t>(kLeastShare, (tokens + shares - 1) / shares);
}

static int64_t sum_shares(int64_t tokens, int64_t width)
{
    const int64_t share = sum_share(tokens, width);
    return (tokens + share - 1) / share;
}

static size_t sorted_bytes(int64_t tokens) { return round_up(static_cast<size_t>(tokens) * sizeof(uint2), 256); }

static bool type_ok(int dtype) { return dtype == MXFP4_OUT_BF16 || dtype == MXFP4_OUT_FP32; }

static int rows_check(const void* a, int64_t ld_a, const void* b, int64_t ld_b, int64_t tokens, int64_t width, int64_t vocab)
{
    if (tokens <= 0 || width <= 0 || vocab <= 0 || width % 8 != 0 || tokens > 0x3FFFFFFF || width > 0x3FFFFFFF ||
        vocab > 0x3FFFFFFF || ld_a < width || ld_b < width)
        return MXFP4_ERR_SHAPE;
    if (!aligned16(a) || !aligned16(b) || ld_a % 8 != 0 || ld_b % 8 != 0) return MXFP4_ERR_ALIGN;
    return MXFP4_OK;
}

int embedding_take_status(int* status) { return take_unit_status(status); }
int embedding_selftest(cudaStream_t st) { return unit_selftest(st); }

}  // namespace mxfp4

using namespace mxfp4;

extern "C" {

int mxfp4_embedding_forward(const int64_t* ids, int64_t tokens, const void* table, int table_dtype, int64_t vocab,
                            int64_t width, int64_t ld_table, float scale, void* out, int out_dtype, int64_t ld_out,
                            void* stream)
{
    if (!ids || !table || !out) return MXFP4_ERR_NULL;
    if (!type_ok(table_dtype) || !type_ok(out_dtype) || !isfinite(scale)) return MXFP4_ERR_ENUM;
    int rc = rows_check(table, ld_table, out, ld_out, tokens, width, vocab);
    if (rc != MXFP4_OK) return rc;
    LookupParams p;
    p.ids = ids;
    p.table = table;
    p.out = out;
    p.ld_table = ld_table;
    p.ld_out = ld_out;
    p.vocab = vocab;
    p.items = tokens * (width / 8);
    p.per_row = static_cast<int32_t>(width / 8);
    p.scale = scale;
    const int64_t blocks = (p.items + kLookupThreads * kLookupUnroll - 1) / (kLookupThreads * kLookupUnroll);
    if (blocks > 0x7FFFFFFF) return MXFP4_ERR_SHAPE;
    if ((rc = device_status_code(device_info())) != MXFP4_OK) return rc;
    const bool in32 = table_dtype == MXFP4_OUT_FP32, out32 = out_dtype == MXFP4_OUT_FP32;
    auto kernel = in32 ? (out32 ? lookup_kernel<float, float> : lookup_kernel<float, __nv_bfloat16>)
                       : (out32 ? lookup_kernel<__nv_bfloat16, float> : lookup_kernel<__nv_bfloat16, __nv_bfloat16>);
    return launch_kernel_pdl(kernel, static_cast<int>(blocks), kLookupThreads, 0, static_cast<cudaStream_t>(stream), p) ==
                   cudaSuccess
               ? MXFP4_OK : MXFP4_ERR_CUDA;
}

size_t mxfp4_embedding_workspace_bytes(int64_t tokens, int64_t vocab, int64_t width)
{
    if (tokens <= 0 || width <= 0 || vocab <= 0 || width % 8 != 0 || tokens > 0x3FFFFFFF || width > 0x3FFFFFFF ||
        vocab > 0x3FFFFFFF)
        return 0;
    return 2 * sorted_bytes(tokens) + round_up(static_cast<size_t>(vocab) * sizeof(uint32_t), 256) +
           static_cast<size_t>(sum_shares(tokens, width)) * 2 * width * sizeof(float);
}

int mxfp4_embedding_backward(const int64_t* ids, int64_t tokens, const void* d_out, int d_out_dtype, int64_t ld_d_out,
                             int64_t vocab, int64_t width, float scale, void* d_table, int d_table_dtype,
                             int64_t ld_d_table, int accumulate, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!ids || !d_out || !d_table) return MXFP4_ERR_NULL;
    if (!type_ok(d_out_dtype) || !type_ok(d_table_dtype) || !isfinite(scale)) return MXFP4_ERR_ENUM;
    int rc = rows_check(d_out, ld_d_out, d_table, ld_d_table, tokens, width, vocab);
    if (rc != MXFP4_OK) return rc;
    const size_t need = mxfp4_embedding_workspace_bytes(tokens, vocab, width);
    if (!workspace || workspace_bytes < need) return MXFP4_ERR_WORKSPACE;
    if (!aligned16(workspace)) return MXFP4_ERR_ALIGN;
    const DeviceInfo& dev = device_info();
    if ((rc = device_status_code(dev)) != MXFP4_OK) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool out32 = d_table_dtype == MXFP4_OUT_FP32, in32 = d_out_dtype == MXFP4_OUT_FP32;
    uint8_t* ws = static_cast<uint8_t*>(workspace);

    SortParams q;
    q.ids = ids;
    q.a = reinterpret_cast<uint2*>(ws);
    q.b = reinterpret_cast<uint2*>(ws + sorted_bytes(tokens));
    q.first = reinterpret_cast<uint32_t*>(ws + 2 * sorted_bytes(tokens));
    q.tokens = static_cast<int32_t>(tokens);
    q.vocab = vocab;
    q.passes = 1;
    while ((vocab >> (kSortBits * q.passes)) != 0) ++q.passes;
    if (tokens <= kRankMost) {
        if (launch_kernel_pdl(rank_kernel, (q.tokens + 31) / 32, kRankWarps * 32, 0, st, q) != cudaSuccess) return MXFP4_ERR_CUDA;
    } else {
        static PerDeviceOnce once;
        const size_t smem = sizeof(SortSmem) + 1024;
        if ((rc = ensure_smem_attribute(once, sort_kernel, smem)) != MXFP4_OK) return rc;
        if (launch_kernel_pdl(sort_kernel, kSortCtas, kSortThreads, smem, st, q) != cudaSuccess) return MXFP4_ERR_CUDA;
    }

    SumParams s;
    s.sorted = q.a;
    s.grads = d_out;
    s.table = d_table;
    s.parts = reinterpret_cast<float*>(ws + 2 * sorted_bytes(tokens) + round_up(static_cast<size_t>(vocab) * sizeof(uint32_t), 256));
    s.ld_grads = ld_d_out;
    s.ld_table = ld_d_table;
    s.tokens = q.tokens;
    s.width = static_cast<int32_t>(width);
    s.share = static_cast<int32_t>(sum_share(tokens, width));
    s.shares = static_cast<int32_t>(sum_shares(tokens, width));
    s.vocab = static_cast<uint32_t>(vocab);
    s.slabs = static_cast<int32_t>(sum_slabs(width));
    s.accumulate = accumulate != 0;
    s.scale = scale;
    const int64_t units = static_cast<int64_t>(s.shares) * s.slabs;
    rc = in32 ? (out32 ? launch_sums<float, float>(s, units, dev.sm_count, st) : launch_sums<float, __nv_bfloat16>(s, units, dev.sm_count, st))
              : (out32 ? launch_sums<__nv_bfloat16, float>(s, units, dev.sm_count, st)
                       : launch_sums<__nv_bfloat16, __nv_bfloat16>(s, units, dev.sm_count, st));
    if (rc != MXFP4_OK) return rc;
    // zeros for a dense gradient, and rows that span shares
    FillParams f;
    f.first = q.first;
    f.pitch = ld_d_table * (out32 ? 4 : 2);
    f.vectors = static_cast<int32_t>(width * (out32 ? 4 : 2) / 16);
    f.blocks = accumulate ? 0 : static_cast<int32_t>((vocab + kFillRows - 1) / kFillRows);
    f.slabs = static_cast<int32_t>((width + 255) / 256);
    const int64_t joins = s.shares > 1 ? (static_cast<int64_t>(s.shares) * f.slabs + kFillRows - 1) / kFillRows : 0;
    if (f.blocks + joins == 0) return MXFP4_OK;
    auto fill = out32 ? fill_join_kernel<float> : fill_join_kernel<__nv_bfloat16>;
    return launch_kernel_pdl(fill, static_cast<int>(f.blocks + joins), kFillRows * 32, 0, st, s, f) == cudaSuccess ? MXFP4_OK
                                                                                                                : MXFP4_ERR_CUDA;
}

}  // extern "C"
