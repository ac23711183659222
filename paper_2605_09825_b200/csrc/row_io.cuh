// Loads and stores of eight consecutive elements of a row (16 bytes of bf16, 32 of fp32) as four pairs of
// fp32 values, the operands of the packed fp32 instructions.  Streamed tensors pass L1 by.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace mxfp4 {

__device__ __forceinline__ uint4 ld_stream(const void* p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p)
                 : "memory");
    return v;
}

__device__ __forceinline__ void st_stream(void* p, const uint4& v)
{
    asm volatile("st.global.L1::no_allocate.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z),
                 "r"(v.w)
                 : "memory");
}

// the two bf16 values of a word
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// eight bf16 of one 16-byte piece as four pairs
__device__ __forceinline__ void unpack8(const uint4& w, float2 (&v)[4])
{
    v[0] = make_float2(bf16_lo(w.x), bf16_hi(w.x));
    v[1] = make_float2(bf16_lo(w.y), bf16_hi(w.y));
    v[2] = make_float2(bf16_lo(w.z), bf16_hi(w.z));
    v[3] = make_float2(bf16_lo(w.w), bf16_hi(w.w));
}

// a vector every row needs
__device__ __forceinline__ void load8(const float* p, float2 (&v)[4])
{
    const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    v[0] = make_float2(a.x, a.y);
    v[1] = make_float2(a.z, a.w);
    v[2] = make_float2(b.x, b.y);
    v[3] = make_float2(b.z, b.w);
}

__device__ __forceinline__ uint4 pack8(const float2 (&v)[4])
{
    return make_uint4(pack_bf16(v[0].x, v[0].y), pack_bf16(v[1].x, v[1].y), pack_bf16(v[2].x, v[2].y),
                      pack_bf16(v[3].x, v[3].y));
}

__device__ __forceinline__ void store8(__nv_bfloat16* p, const float2 (&v)[4]) { st_stream(p, pack8(v)); }

__device__ __forceinline__ void store8(float* p, const float2 (&v)[4])
{
    st_stream(p, make_uint4(__float_as_uint(v[0].x), __float_as_uint(v[0].y), __float_as_uint(v[1].x), __float_as_uint(v[1].y)));
    st_stream(p + 4, make_uint4(__float_as_uint(v[2].x), __float_as_uint(v[2].y), __float_as_uint(v[3].x), __float_as_uint(v[3].y)));
}

// rounds to bf16, stores and leaves the stored values in v (fp32: stores)
__device__ __forceinline__ void store8_round(__nv_bfloat16* p, float2 (&v)[4], bool store)
{
    const uint4 w = pack8(v);
    if (store) st_stream(p, w);
    unpack8(w, v);
}
__device__ __forceinline__ void store8_round(float* p, float2 (&v)[4], bool store)
{
    if (store) store8(p, v);
}

__device__ __forceinline__ float2 pair(float v) { return make_float2(v, v); }

}  // namespace mxfp4
