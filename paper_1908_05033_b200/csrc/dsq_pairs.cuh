// Two binary32 values in a pair of registers, worked on by one instruction (sm_100a's f32x2: each half
// rounds as the scalar operation does; half the issue slots).
#pragma once

#include <stdint.h>

typedef unsigned long long DsqPair;

__device__ __forceinline__ DsqPair dsq_pair_of(float a, float b)
{
    DsqPair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void dsq_halves(DsqPair v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ DsqPair dsq_pair_add(DsqPair a, DsqPair b)
{
    DsqPair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ DsqPair dsq_pair_mul(DsqPair a, DsqPair b)
{
    DsqPair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ DsqPair dsq_pair_fma(DsqPair a, DsqPair b, DsqPair c)
{
    DsqPair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ DsqPair dsq_pair_neg(DsqPair a) { return a ^ 0x8000000080000000ull; }
