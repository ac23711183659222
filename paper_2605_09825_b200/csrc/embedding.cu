// Token embeddings: scaled lookup, and the gradient of the table (see include/mxfp4.h).
//
// Backward, three launches:
//   1. the first cluster sorts the token ids (below) while all other CTAs set the rows that no token has to zero, which
//      for a large vocabulary is most of the bytes: a CTA learns which of its rows those are by reading all ids;
//   2. sums: the sorted positions in chunks, a warp per chunk and 256 columns, gradients added in fp32 in the order of
//      their positions; a row whose positions all lie in one chunk is written at once, a part of a row that goes on
//      in another chunk becomes a partial sum;
//   3. partial sums are joined in the order of their chunks.
// No floating-point atomics: results depend on the inputs alone.
//
// The sort: a cluster of eight CTAs, 9 bits per pass from the lowest.  Each CTA counts the digits of its eighth of the
// positions, reads the other CTAs' counts through distributed shared memory and places its positions, 1024 at a time,
// behind the smaller digits, the earlier CTAs' and its own earlier ones: equal ids stay in the order of their
// positions.  Ids without a row sort behind all others.
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

// ------------------------------------------------------------------ sort and rows without tokens
constexpr int kSortCtas = 8;                       // one cluster
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortBits = 9;
constexpr int kSortBins = 1 << kSortBits;
constexpr int kFillRows = 1 << 16;                 // rows a CTA looks up at a time

struct SortParams {
    const int64_t* ids;
    uint2* a;                    // (id, position), in turn source and destination; the result is in a
    uint2* b;
    int32_t tokens;
    int32_t passes;
    int64_t vocab;
    // rows without tokens
    uint8_t* table;
    int64_t pitch;               // bytes
    int32_t row_vectors;         // 16-byte pieces per row
};

struct SortSmem {
    uint32_t counts[kSortBins];                    // of this CTA's positions
    uint32_t start[kSortBins];                     // where the next position with this digit goes
    uint32_t warp_counts[kSortWarps][kSortBins];   // digits of a round, then where each warp's start
    uint32_t sums[kSortWarps];
};

union SortFillSmem {
    SortSmem sort;
    uint32_t touched[kFillRows / 32];
};

__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t cluster_addr)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_addr) : "memory");
    return v;
}

__device__ void sort_ids(const SortParams& p, SortSmem& s, uint32_t rank)
{
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    const int share = (p.tokens + kSortCtas - 1) / kSortCtas;
    const int begin = min(p.tokens, static_cast<int>(rank) * share), end = min(p.tokens, begin + share);
    const uint2* from = nullptr;
    for (int pass = 0; pass < p.passes; ++pass) {
        uint2* to = (p.passes - pass) & 1 ? p.a : p.b;
        const int shift = pass * kSortBits;
        auto entry = [&](int i) {
            if (from) return from[i];
            const int64_t id = p.ids[i];
            return make_uint2(static_cast<uint32_t>(id < 0 || id >= p.vocab ? p.vocab : id), static_cast<uint32_t>(i));
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
        // 1024 positions at a time
        for (int i0 = begin; i0 < end; i0 += kSortThreads) {
            for (int i = t; i < kSortWarps * kSortBins; i += kSortThreads) smem_store(&s.warp_counts[0][0] + i, 0u, s.warp_counts, sizeof(s.warp_counts));
            __syncthreads();
            const int i = i0 + t;
            const bool in = i < end;
            const uint2 e = in ? entry(i) : make_uint2(0u, 0u);
            const int d = digit_of(e);
            // lanes with the same digit (those past the end among themselves)
            const uint32_t same = __match_any_sync(0xffffffffu, in ? d : kSortBins + lane);
            const int ahead = __popc(same & ((1u << lane) - 1));
            if (in && ahead == 0) smem_store(&s.warp_counts[warp][d], static_cast<uint32_t>(__popc(same)), s.warp_counts, sizeof(s.warp_counts));
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
            if (in) {
                const uint32_t at = smem_load<uint32_t>(&s.warp_counts[warp][d], s.warp_counts, sizeof(s.warp_counts)) + ahead;
                if (at < static_cast<uint32_t>(p.tokens)) to[at] = e;
            }
            __syncthreads();
        }
        cluster_sync_all();      // everything is placed, and the counts have been read
        from = to;
    }
}

__device__ void fill_rows(const SortParams& p, uint32_t (&touched)[kFillRows / 32], int cta, int ctas)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t share = (p.vocab + ctas - 1) / ctas;
    const int64_t last = min(p.vocab, (cta + 1) * share);
    for (int64_t v0 = cta * share; v0 < last; v0 += kFillRows) {
        const int rows = static_cast<int>(min(last - v0, static_cast<int64_t>(kFillRows)));
        for (int i = threadIdx.x; i < (rows + 31) / 32; i += kSortThreads) smem_put(touched, i, 0u);
        __syncthreads();
        for (int i = threadIdx.x; i < p.tokens; i += kSortThreads) {
            const int64_t r = p.ids[i] - v0;
            if (r >= 0 && r < rows && smem_within(touched, static_cast<int>(r >> 5)))
                atomicOr(touched + (r >> 5), 1u << (r & 31));
        }
        __syncthreads();
        for (int r = warp; r < rows; r += kSortWarps) {
            if (smem_get(touched, r >> 5) >> (r & 31) & 1) continue;
            uint8_t* to = p.table + (v0 + r) * p.pitch;
            for (int i = lane; i < p.row_vectors; i += 32) st_stream(to + i * 16, make_uint4(0u, 0u, 0u, 0u));
        }
        __syncthreads();
    }
}

__global__ void __cluster_dims__(kSortCtas, 1, 1) __launch_bounds__(kSortThreads, 2) sort_fill_kernel(const __grid_constant__ SortParams p)
{
    extern __shared__ uint8_t smem_raw[];
    SortFillSmem& sm = *reinterpret_cast<SortFillSmem*>(smem_align_1024(smem_raw));
    griddep_launch_dependents();
    griddep_wait();
    if (blockIdx.x < kSortCtas) sort_ids(p, sm.sort, cluster_ctarank());
    else fill_rows(p, sm.touched, blockIdx.x - kSortCtas, gridDim.x - kSortCtas);
}

// ------------------------------------------------------------------ sums
struct SumParams {
    const uint2* sorted;         // (id, position)
    const void* grads;
    void* table;
    float* parts;                // [chunk][first, last][width]
    int64_t ld_grads, ld_table;
    int32_t tokens, width;
    int32_t chunk;               // positions per chunk
    int32_t chunks;
    uint32_t vocab;
    int32_t slabs;               // pieces of 256 columns
    int32_t accumulate;
    float scale;
};

constexpr int kSumWarps = 8;
constexpr int kSumUnroll = 8;    // rows in flight per warp

template <class Out>
__device__ __forceinline__ void write_row(const SumParams& p, uint32_t id, int col, float2 (&acc)[4])
{
    Out* to = static_cast<Out*>(p.table) + id * p.ld_table + col;
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = make_float2(acc[j].x * p.scale, acc[j].y * p.scale);
    if (p.accumulate) {
        float2 old[4];
        load8_stream(to, old);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = make_float2(acc[j].x + old[j].x, acc[j].y + old[j].y);
    }
    store8(to, acc);
}

// A chunk's first row, where earlier chunks have positions of it too, is a partial sum in slot 0; its last row, where it
// begins here and goes on in later chunks, in slot 1.
template <class In, class Out>
__global__ void __launch_bounds__(kSumWarps * 32) sum_kernel(const SumParams p)
{
    griddep_launch_dependents();
    griddep_wait();
    const int64_t work = static_cast<int64_t>(blockIdx.x) * kSumWarps + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    const int chunk = static_cast<int>(work / p.slabs);
    if (chunk >= p.chunks) return;
    const int col = (static_cast<int>(work - static_cast<int64_t>(chunk) * p.slabs) * 32 + lane) * 8;
    const bool col_ok = col < p.width;
    const int begin = chunk * p.chunk, end = min(p.tokens, begin + p.chunk);
    const uint32_t before = begin > 0 ? p.sorted[begin - 1].x : 0xFFFFFFFFu;
    const uint32_t after = end < p.tokens ? p.sorted[end].x : 0xFFFFFFFFu;
    float2 acc[4];
    uint32_t id = p.sorted[begin].x;
    bool fresh = true;           // nothing of `id` added yet
    bool first = true;           // `id` is the chunk's first
    auto finish = [&](bool last) {
        if (!col_ok || id >= p.vocab) return;
        if (first && id == before) store8(p.parts + (static_cast<int64_t>(chunk) * 2) * p.width + col, acc);
        else if (last && id == after) store8(p.parts + (static_cast<int64_t>(chunk) * 2 + 1) * p.width + col, acc);
        else write_row<Out>(p, id, col, acc);
    };
    for (int i0 = begin; i0 < end; i0 += kSumUnroll) {
        uint2 e[kSumUnroll];
        float2 v[kSumUnroll][4];
#pragma unroll
        for (int u = 0; u < kSumUnroll; ++u) e[u] = i0 + u < end ? p.sorted[i0 + u] : make_uint2(p.vocab, 0u);
#pragma unroll
        for (int u = 0; u < kSumUnroll; ++u) {
            if (col_ok && e[u].x < p.vocab)
                load8_stream(static_cast<const In*>(p.grads) + e[u].y * p.ld_grads + col, v[u]);
        }
#pragma unroll
        for (int u = 0; u < kSumUnroll; ++u) {
            if (i0 + u >= end) break;
            if (e[u].x != id) {
                finish(false);
                id = e[u].x;
                fresh = true;
                first = false;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                acc[j] = fresh ? v[u][j] : make_float2(acc[j].x + v[u][j].x, acc[j].y + v[u][j].y);
            fresh = false;
        }
    }
    finish(true);
}

// Rows that span chunks, from the chunk they begin in.
template <class Out>
__global__ void __launch_bounds__(kSumWarps * 32) sum_join_kernel(const SumParams p)
{
    griddep_launch_dependents();
    griddep_wait();
    const int64_t work = static_cast<int64_t>(blockIdx.x) * kSumWarps + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    const int chunk = static_cast<int>(work / p.slabs);
    if (chunk + 1 >= p.chunks) return;
    const int col = (static_cast<int>(work - static_cast<int64_t>(chunk) * p.slabs) * 32 + lane) * 8;
    const int begin = chunk * p.chunk;
    const uint32_t id = p.sorted[begin + p.chunk].x;
    // it goes on in the next chunk, and begins in this one
    if (id >= p.vocab || p.sorted[begin + p.chunk - 1].x != id || (begin > 0 && p.sorted[begin - 1].x == id)) return;
    if (col >= p.width) return;
    float2 acc[4];
    load8_stream(p.parts + (static_cast<int64_t>(chunk) * 2 + 1) * p.width + col, acc);
    for (int c = chunk + 1; c < p.chunks && p.sorted[c * p.chunk].x == id; ++c) {
        float2 v[4];
        load8_stream(p.parts + (static_cast<int64_t>(c) * 2) * p.width + col, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = make_float2(acc[j].x + v[j].x, acc[j].y + v[j].y);
    }
    write_row<Out>(p, id, col, acc);
}

// Positions per chunk: few enough that the device is full at some thousand tokens, and not more than 4096 chunks, so that
// a token that is most of a long text has not too many partial sums to join.
static int64_t sum_chunk(int64_t tokens)
{
    const int64_t c = (tokens + 4095) / 4096;
    return c < 32 ? 32 : (c + 31) / 32 * 32;
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

size_t mxfp4_embedding_workspace_bytes(int64_t tokens, int64_t width)
{
    if (tokens <= 0 || width <= 0 || width % 8 != 0 || tokens > 0x3FFFFFFF || width > 0x3FFFFFFF) return 0;
    const int64_t chunk = sum_chunk(tokens), chunks = (tokens + chunk - 1) / chunk;
    return 2 * sorted_bytes(tokens) + static_cast<size_t>(chunks) * 2 * width * sizeof(float);
}

int mxfp4_embedding_backward(const int64_t* ids, int64_t tokens, const void* d_out, int d_out_dtype, int64_t ld_d_out,
                             int64_t vocab, int64_t width, float scale, void* d_table, int d_table_dtype,
                             int64_t ld_d_table, int accumulate, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!ids || !d_out || !d_table) return MXFP4_ERR_NULL;
    if (!type_ok(d_out_dtype) || !type_ok(d_table_dtype) || !isfinite(scale)) return MXFP4_ERR_ENUM;
    int rc = rows_check(d_out, ld_d_out, d_table, ld_d_table, tokens, width, vocab);
    if (rc != MXFP4_OK) return rc;
    const size_t need = mxfp4_embedding_workspace_bytes(tokens, width);
    if (!workspace || workspace_bytes < need) return MXFP4_ERR_WORKSPACE;
    if (!aligned16(workspace)) return MXFP4_ERR_ALIGN;
    SumParams s;
    s.slabs = static_cast<int32_t>((width + 255) / 256);
    s.chunk = static_cast<int32_t>(sum_chunk(tokens));
    s.chunks = static_cast<int32_t>((tokens + s.chunk - 1) / s.chunk);
    const int64_t blocks = (static_cast<int64_t>(s.chunks) * s.slabs + kSumWarps - 1) / kSumWarps;
    if (blocks > 0x7FFFFFFF) return MXFP4_ERR_SHAPE;
    const DeviceInfo& dev = device_info();
    if ((rc = device_status_code(dev)) != MXFP4_OK) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool out32 = d_table_dtype == MXFP4_OUT_FP32, in32 = d_out_dtype == MXFP4_OUT_FP32;

    SortParams q;
    q.ids = ids;
    q.a = static_cast<uint2*>(workspace);
    q.b = reinterpret_cast<uint2*>(static_cast<uint8_t*>(workspace) + sorted_bytes(tokens));
    q.tokens = static_cast<int32_t>(tokens);
    q.vocab = vocab;
    q.passes = 1;
    while ((vocab >> (kSortBits * q.passes)) != 0) ++q.passes;
    q.table = static_cast<uint8_t*>(d_table);
    q.pitch = ld_d_table * (out32 ? 4 : 2);
    q.row_vectors = static_cast<int32_t>(width * (out32 ? 4 : 2) / 16);
    static PerDeviceOnce once;
    const size_t smem = sizeof(SortFillSmem) + 1024;
    if ((rc = ensure_smem_attribute(once, sort_fill_kernel, smem)) != MXFP4_OK) return rc;
    // two CTAs of 1024 threads per SM
    const int fill = accumulate ? 0 : 2 * (dev.sm_count / kSortCtas) - 1;
    if (launch_kernel_pdl(sort_fill_kernel, kSortCtas * (1 + fill), kSortThreads, smem, st, q) != cudaSuccess)
        return MXFP4_ERR_CUDA;

    s.sorted = q.a;
    s.grads = d_out;
    s.table = d_table;
    s.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + 2 * sorted_bytes(tokens));
    s.ld_grads = ld_d_out;
    s.ld_table = ld_d_table;
    s.tokens = q.tokens;
    s.width = static_cast<int32_t>(width);
    s.vocab = static_cast<uint32_t>(vocab);
    s.accumulate = accumulate != 0;
    s.scale = scale;
    auto sum = in32 ? (out32 ? sum_kernel<float, float> : sum_kernel<float, __nv_bfloat16>)
                    : (out32 ? sum_kernel<__nv_bfloat16, float> : sum_kernel<__nv_bfloat16, __nv_bfloat16>);
    if (launch_kernel_pdl(sum, static_cast<int>(blocks), kSumWarps * 32, 0, st, s) != cudaSuccess) return MXFP4_ERR_CUDA;
    if (s.chunks == 1) return MXFP4_OK;
    auto join = out32 ? sum_join_kernel<float> : sum_join_kernel<__nv_bfloat16>;
    return launch_kernel_pdl(join, static_cast<int>(blocks), kSumWarps * 32, 0, st, s) == cudaSuccess ? MXFP4_OK
                                                                                                      : MXFP4_ERR_CUDA;
}

}  // extern "C"
