// Storage types of the operators that take more than one (dsq_dtype): eight
// consecutive elements as binary32 values, and one element.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "dsq_common.cuh"

static inline bool dsq_is_float_type(int dtype)
{
    return dtype == DSQ_F32 || dtype == DSQ_BF16 || dtype == DSQ_F16;
}

#ifdef __CUDACC__
__device__ __forceinline__ float dsq_to_f32(float v) { return v; }
__device__ __forceinline__ float dsq_to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float dsq_to_f32(__half v) { return __half2float(v); }

// to nearest, ties to even: the only rounding of an output to its type
template <class T> __device__ __forceinline__ T dsq_from_f32(float v);
template <> __device__ __forceinline__ float dsq_from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 dsq_from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half dsq_from_f32<__half>(float v) { return __float2half_rn(v); }

// eight elements at an address that is a multiple of their size (16 or 32 bytes), as
// they lie in memory
template <class T> struct alignas(16) DsqRaw8 { uint4 v[sizeof(T) * 8 / 16]; };

// (ld.global, not the read-only path: an output may be the buffer of an input)
template <class T> __device__ __forceinline__ DsqRaw8<T> dsq_load8(const T *p)
{
    DsqRaw8<T> r;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(r) / 16); ++i)
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(r.v[i].x), "=r"(r.v[i].y), "=r"(r.v[i].z), "=r"(r.v[i].w)
                     : "l"(reinterpret_cast<const uint4 *>(p) + i));
    return r;
}
template <class T> __device__ __forceinline__ void dsq_store8(T *p, const DsqRaw8<T> &r)
{
#pragma unroll
    for (int i = 0; i < (int)(sizeof(r) / 16); ++i) reinterpret_cast<uint4 *>(p)[i] = r.v[i];
}

__device__ __forceinline__ void dsq_unpack8(const DsqRaw8<float> &r, float (&f)[8])
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        f[4 * i] = __uint_as_float(r.v[i].x); f[4 * i + 1] = __uint_as_float(r.v[i].y);
        f[4 * i + 2] = __uint_as_float(r.v[i].z); f[4 * i + 3] = __uint_as_float(r.v[i].w);
    }
}
__device__ __forceinline__ void dsq_unpack8(const DsqRaw8<__nv_bfloat16> &r, float (&f)[8])
{
    const uint32_t w[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void dsq_unpack8(const DsqRaw8<__half> &r, float (&f)[8])
{
    const uint32_t w[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
        f[2 * i] = v.x;
        f[2 * i + 1] = v.y;
    }
}
__device__ __forceinline__ void dsq_pack8(const float (&f)[8], DsqRaw8<float> &r)
{
#pragma unroll
    for (int i = 0; i < 2; ++i)
        r.v[i] = make_uint4(__float_as_uint(f[4 * i]), __float_as_uint(f[4 * i + 1]),
                            __float_as_uint(f[4 * i + 2]), __float_as_uint(f[4 * i + 3]));
}
__device__ __forceinline__ uint32_t dsq_pair(float a, float b, __nv_bfloat16)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t dsq_pair(float a, float b, __half)
{
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <class T> __device__ __forceinline__ void dsq_pack8(const float (&f)[8], DsqRaw8<T> &r)
{
    r.v[0] = make_uint4(dsq_pair(f[0], f[1], T()), dsq_pair(f[2], f[3], T()),
                        dsq_pair(f[4], f[5], T()), dsq_pair(f[6], f[7], T()));
}
#endif
