// What the kernels for products with group-wise 4-bit weights share (dsq_wgemm_group.cu: mma.sync;
// dsq_wgemm_group_few.cu: mma.sync on digits, one or two rows; dsq_wgemm_group_tc.cu: tcgen05).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "dsq_launch.h"
#include "dsq_types.cuh"

struct DsqGroupGemm {
    const uint8_t *X, *W;
    const float *scales, *bias, *row_scale;
    void *Y;
    int64_t N;
    int M, K, pitch;              // pitch: bytes of a row of codes
    int groups;
    uint32_t units, units_inv;    // of 32 x pieces codes in a group, floor(2^32 / units) + 1
    int odd;                      // values 2 c + 1 (else c)
    int y_type;

    void set_units(int64_t group, int pieces)
    {
        units = (uint32_t)(group / (32 * pieces));
        units_inv = units > 1 ? (uint32_t)((1ull << 32) / units + 1) : 0u;
    }
#ifdef __CUDACC__
    // group of a unit (both below 2^15 + 4: the product with the rounded-up inverse is exact enough)
    __device__ __forceinline__ int group_of(uint32_t unit) const
    {
        return units == 1 ? (int)unit : (int)__umulhi(unit, units_inv);
    }
    __device__ __forceinline__ void store(int m, int64_t n, float s) const
    {
        if (row_scale) s *= __ldg(row_scale + m);
        if (bias) s += __ldg(bias + n);
        const int64_t to = (int64_t)m * N + n;
        if (y_type == DSQ_F32) ((float *)Y)[to] = s;
        else if (y_type == DSQ_BF16) ((__nv_bfloat16 *)Y)[to] = __float2bfloat16_rn(s);
        else ((__half *)Y)[to] = __float2half_rn(s);
    }
#endif
};

// pieces of 32 codes, up to four, that no group's end cuts
static inline int dsq_group_pieces(int64_t group) { return group % 128 == 0 ? 4 : group % 64 == 0 ? 2 : 1; }

// Arguments validated; group a multiple of 32.
// tcgen05 (est_us: its estimated time is written there and nothing is launched)
DSQ_HIDDEN int dsq_wgemm_group_tc(const DsqGroupGemm &p, int x_type, int64_t group, cudaStream_t s, double *est_us);
// one or two rows in 16 bits
DSQ_HIDDEN int dsq_wgemm_group_few(const DsqGroupGemm &p, int x_type, int64_t group, cudaStream_t s);

#ifdef __CUDACC__
// codes i and i + 4 of a word as a pair of 16-bit values (2 c + 1) / 32 or c / 16: the field in the
// upper mantissa bits of 1.0 is 1 + q / 16 (q = c + 8), less 1 + 7.5 / 16 or 1.5
template <int XT> __device__ __forceinline__ uint32_t dsq_value_base(int odd)
{
    return XT == DSQ_BF16 ? (odd ? 0x3FBC3FBCu : 0x3FC03FC0u) : (odd ? 0x3DE03DE0u : 0x3E003E00u);
}
template <int XT> __device__ __forceinline__ uint32_t dsq_value_pair(uint32_t w, int i, uint32_t base)
{
    constexpr int AT = XT == DSQ_BF16 ? 3 : 6;                // the field's place in the mantissa
    constexpr uint32_t MASK = (0xFu << AT) * 0x00010001u;
    constexpr uint32_t FLIP = ((XT == DSQ_BF16 ? 0x3F80u : 0x3C00u) ^ (8u << AT)) * 0x00010001u;
    const uint32_t y = 4 * i > AT ? w >> (4 * i - AT) : w << (AT - 4 * i);
    uint32_t v;                       // (y & MASK) ^ FLIP: as C, with two constants, it is two instructions
    asm("lop3.b32 %0, %1, %2, %3, 0x6a;" : "=r"(v) : "r"(y), "r"(MASK), "r"(FLIP));
    if (XT == DSQ_BF16) {
        const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&v),
                                         *reinterpret_cast<const __nv_bfloat162 *>(&base));
        return *reinterpret_cast<const uint32_t *>(&r);
    }
    const __half2 r = __hsub2(*reinterpret_cast<const __half2 *>(&v), *reinterpret_cast<const __half2 *>(&base));
    return *reinterpret_cast<const uint32_t *>(&r);
}
// what sums are multiples of: int8 values are 8 (2 c + 1) or 16 c
template <int XT> __device__ __forceinline__ float dsq_value_unit(int odd)
{
    return XT == DSQ_I8 ? (odd ? 0.125f : 0.0625f) : (odd ? 32.f : 16.f);
}

// instruction descriptor for kind::f16 with fp16 operands and an f32 accumulator
__device__ __forceinline__ uint32_t dsq_idesc_f16(int n)
{
    return 1u << 4 | (uint32_t)(n >> 3) << 17 | 8u << 24;
}
__device__ __forceinline__ uint2 lds_64(uint32_t at)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t ld_cluster_32(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
#endif
