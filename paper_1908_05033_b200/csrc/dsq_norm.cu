// Root-mean-square norm in front of a low-bit linear layer, and its backward pass.
//
//   h = x + residual;  rstd = 1/sqrt(mean_k h^2 + eps);  y = h rstd w
//   8 bits: a = max_k |h w|, q = floor(127 h w / a + 1/2), s = rstd a / 127 (so that
//   y is about s q): the codes do not depend on rstd, and one pass of reductions
//   gives the sum of squares and a together.  Codes are exact for the h and w that binary32
//   holds: a code on the wrong side of a border changes every output of the product behind it.
//   The reductions bring what the rounding of a lost as well, and elements next to a border
//   are decided with what theirs lost (nothing at 8192 x 4096 in bf16, where memory
//   binds; of shorter and unaligned rows, where instructions do, up to a quarter: 16384 x 1024 23.7 -> 29.9 us).
//   backward, with g = grad_y w and n = h rstd:
//   grad_x = rstd (g - n mean_k(g n)) + grad_h,  grad_w = sum_m grad_y n
//
// All arithmetic is binary32; outputs are rounded once, to their type.  The sum of the
// residual is not rounded before it is normalised.  Rows whose squares overflow, or vanish beside
// a tiny eps, take a second reduction of the row times a power of two.
//
// Bound: memory (bf16: 8 bytes an element forward with residual, 8 backward): 8192 x 4096 in bf16 takes
// 44.4 us forward with fake-quantised output (0.93 of the copy's rate) and 49 backward (0.84; 45 without
// grad_w, whose sums over the blocks are a kernel of their own).  A row stays in
// registers between its reduction and its outputs, so every input is read once; the next
// row of the same threads is on its way meanwhile.  Rows whose length is no multiple of
// eight start inside a 16-byte vector: the eight-element vectors are counted from the
// start of the array then, which is the same grid for all arrays of one shape whatever
// their types, and the up to 14 elements in front of a row's first whole vector and behind
// its last go one by one, a thread each.  (With those vectors read whole and masked
// every element paid: 8888 x 1777 backward 35 us, 4096 x 5001 96.)
// A thread meets the same columns in all its rows (the weight, and the sums of grad_w,
// stay in registers): its rows are a multiple of eight apart where rows shift.
#include <math.h>

#include <type_traits>

#include "dsq_launch.h"
#include "dsq_ptx.cuh"
#include "dsq_tc_host.h"
#include "dsq_types.cuh"

using dsq_ptx::grid_dependency_wait;
using dsq_ptx::grid_launch_dependents;

namespace {

constexpr int64_t MAX_K = 49152;          // the backward pass keeps a row of sums in shared memory

struct FwdParams {
    const void *x, *res;
    const float *w;
    void *h, *y;
    int8_t *codes;
    float *scale, *rstd;
    int64_t M;
    int K;
    float eps, inv_k;
};
struct BwdParams {
    const void *gy, *gh, *h;
    const float *w, *rstd;
    void *gx;
    float *part;                          // [blocks][K], or NULL
    int64_t M;
    int K;
    float inv_k;
};

__host__ __device__ constexpr int block_of(int tpr) { return tpr < 256 ? 256 : tpr; }

// Where a row's elements lie that are `shift` behind a multiple of eight from the array's start:
// `head` single ones, nv vectors, single ones again.  ALIGNED: vectors only.
struct Cut { int head, nv, singles; };
template <bool ALIGNED> __device__ __forceinline__ Cut cut_of(int64_t row, int K)
{
    if (ALIGNED) return {0, K >> 3, 0};
    const int shift = ((int)(row & 7) * (K & 7)) & 7, head = min((8 - shift) & 7, K);
    const int nv = (K - head) >> 3;
    return {head, nv, K - 8 * nv};
}
// column of single element j
__device__ __forceinline__ int single_of(const Cut &c, int j) { return j < c.head ? j : j + 8 * c.nv; }

// the low bytes of eight numbers
__device__ __forceinline__ void store_codes(int8_t *p, const float (&f)[8])
{
    uint2 v;
    const auto u = [&](int i) { return __float_as_uint(f[i]); };
    v.x = __byte_perm(__byte_perm(u(0), u(1), 0x0040), __byte_perm(u(2), u(3), 0x0040), 0x5410);
    v.y = __byte_perm(__byte_perm(u(4), u(5), 0x0040), __byte_perm(u(6), u(7), 0x0040), 0x5410);
    *reinterpret_cast<uint2 *>(p) = v;
}
template <class T> __device__ __forceinline__ void store_vec(T *p, const float (&f)[8])
{
    DsqRaw8<T> r;
    dsq_pack8(f, r);
    dsq_store8(p, r);
}
template <bool ALIGNED>
__device__ __forceinline__ void load_weight(const float *w, bool in, float (&f)[8])
{
    if (ALIGNED && in) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float4 v = __ldg(reinterpret_cast<const float4 *>(w) + i);
            f[4 * i] = v.x; f[4 * i + 1] = v.y; f[4 * i + 2] = v.z; f[4 * i + 3] = v.w;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = in ? __ldg(w + i) : 0.f;
}

// sum and largest of the TPR threads of a row, to all of them.  `red`: one entry a warp.
// Every thread of the block calls it.
template <int TPR>
__device__ __forceinline__ void reduce_row(float &sum, uint32_t &top, float2 *red)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
    for (int o = (TPR < 32 ? TPR : 32) / 2; o > 0; o >>= 1) {
        sum += __shfl_xor_sync(~0u, sum, o);
        if (TPR < 32) top = max(top, __shfl_xor_sync(~0u, top, o));
    }
    if (TPR >= 32) top = __reduce_max_sync(~0u, top);
    if constexpr (TPR > 32) {
        constexpr int W = TPR / 32;
        if (lane == 0) red[warp] = make_float2(sum, __uint_as_float(top));
        __syncthreads();
        const float2 v = red[warp / W * W + (lane % W)];
        sum = v.x;
#pragma unroll
        for (int o = W / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
        top = __reduce_max_sync(~0u, __float_as_uint(v.y));
    }
}

// What the rounding of the largest |h w| lost: the largest |h w| - top, exactly (times 2^60 where top is so small that
// some of it would lie below binary32's smallest number), as bits that order like numbers and are never 0.
constexpr float SMALL = 8.6736174e-19f, UP = 1.1529215e18f;     // 2^-60, 2^60
// the largest of three, NaN where one is
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
template <bool TINY> __device__ __forceinline__ float above(float most, float h, float w, float top)
{
    if (!TINY) return max3(most, __fmaf_rn(h, w, -top), __fmaf_rn(-h, w, -top));
    const float ah = fabsf(h), aw = fabsf(w);
    return fmaxf(most, __fmaf_rn(fminf(ah, aw) * UP, fmaxf(ah, aw), -top * UP));
}
// largest |h w| of N elements and `most`
template <int N> __device__ __forceinline__ float largest(float most, const float (&h)[N], const float (&w)[N])
{
#pragma unroll
    for (int k = 0; k + 1 < N; k += 2) most = max3(most, fabsf(h[k] * w[k]), fabsf(h[k + 1] * w[k + 1]));
    if (N % 2) most = max3(most, most, fabsf(h[N - 1] * w[N - 1]));
    return most;
}
__device__ __forceinline__ uint32_t ordered(float v)
{
    const uint32_t bits = __float_as_uint(v);
    return bits ^ ((uint32_t)((int)bits >> 31) | 0x80000000u);
}

__device__ __forceinline__ float from_ordered(uint32_t v) { return __uint_as_float((int)v < 0 ? v ^ 0x80000000u : ~v); }
template <int N> __device__ __forceinline__ uint32_t low_of(const float (&h)[N], const float (&w)[N], float own)
{
    float most = -INFINITY;
#pragma unroll
    for (int i = 0; i < N; ++i) most = own >= SMALL ? above<false>(most, h[i], w[i], own) : above<true>(most, h[i], w[i], own);
    return ordered(most);
}

// Whether a mean of squares (and eps) has left binary32's range, or is so small that squares below it count.
__device__ __forceinline__ bool out_of_range(float mean) { return !(mean < 3.0e38f) || mean < 8.2718061e-25f; }     // 2^-80

// The same for the forward pass, where the largest is wanted for rows in 8 bits alone, and with it what its rounding lost:
// the largest `low` of the threads that have it.  True, for all threads that share a barrier, where the sum of one of their
// rows is out of range.
template <int TPR, bool EIGHT>
__device__ __forceinline__ bool reduce_row_low(float &sum, uint32_t &top, uint32_t &low, float4 *red, float inv_k, float eps)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    [[maybe_unused]] const uint32_t own = top;
#pragma unroll
    for (int o = (TPR < 32 ? TPR : 32) / 2; o > 0; o >>= 1) {
        sum += __shfl_xor_sync(~0u, sum, o);
        if (EIGHT && TPR < 32) top = max(top, __shfl_xor_sync(~0u, top, o));
    }
    if constexpr (EIGHT) {
        if (TPR >= 32) top = __reduce_max_sync(~0u, top);
        low = own == top ? low : 0u;
        if (TPR >= 32) {
            low = __reduce_max_sync(~0u, low);
        } else {
#pragma unroll
            for (int o = TPR / 2; o > 0; o >>= 1) low = max(low, __shfl_xor_sync(~0u, low, o));
        }
    }
    bool far;
    if constexpr (TPR > 32) {
        constexpr int W = TPR / 32, ALL = block_of(TPR) / 32;        // warps of a row, of the block
        if (lane == 0) red[warp] = make_float4(sum, __uint_as_float(top), __uint_as_float(low), 0.f);
        __syncthreads();
        const float4 v = red[lane % ALL];
        const bool mine = ALL == W || lane % ALL / W == warp / W;
        sum = v.x;
#pragma unroll
        for (int o = W / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
        far = __any_sync(~0u, out_of_range(__fmaf_rn(sum, inv_k, eps)));
        if (ALL > W) sum = __shfl_sync(~0u, sum, warp / W * W);
        if constexpr (EIGHT) {
            top = __reduce_max_sync(~0u, mine ? __float_as_uint(v.y) : 0u);
            low = __reduce_max_sync(~0u, mine && __float_as_uint(v.y) == top ? __float_as_uint(v.z) : 0u);
        }
    } else {
        far = __any_sync(~0u, out_of_range(__fmaf_rn(sum, inv_k, eps)));
    }
    return far;
}

// 1 / sqrt(mean + eps) of a row whose sum is out of range, from the sum of squares times f^2: 2^-80 where squares are too large, 2^90
// where they are too small.
__device__ __forceinline__ float far_factor(float sum, float inv_k, float eps)
{
    return __fmaf_rn(sum, inv_k, eps) < 1.f ? 1.2379401e27f : 8.2718061e-25f;
}
__device__ __forceinline__ float far_rstd(float sum, float f, float inv_k, float eps)
{
    const float mean = __fmaf_rn(sum, inv_k, eps * f * f);
    // (a row of zeros with eps = 0: 0, so that its outputs are)
    const float r = mean == 0.f ? 0.f : __fdiv_rn(f, __fsqrt_rn(mean));
    return r > 3.4028235e38f ? 3.4028235e38f : r;            // (NaN stays)
}

// what a row's reductions give its elements
struct RowQuant { float rstd, inv, up, s; uint32_t top, low; };      // inv, up: 127 / a, less and more a small part of it
__device__ __forceinline__ RowQuant row_quant(float rstd, uint32_t top, uint32_t low)
{
    RowQuant r;
    r.rstd = rstd;
    const float a = __uint_as_float(top);
    // (bits above those of infinity: NaN)
    const bool bad = top >= 0x7F800000u, none = a < 1.5046328e-36f;      // 2^-119: 127 / a is finite
    // 127 / (a and what its rounding lost), rounded once
    const float quot = __fdiv_rn(127.f, a), low_part = from_ordered(low) * (a < SMALL ? 1.f / UP : 1.f);
    const float inv = __fmaf_rn(-quot, low_part * quot * (1.f / 127.f), quot);
    const float part = a < SMALL ? 3.8146973e-6f : 2.3841858e-7f;       // 2^-18 (products lose more bits there), 2^-22
    r.inv = bad || none ? 0.f : inv * (1.f - part);
    r.up = inv * (1.f + part);
    r.s = bad ? __uint_as_float(0x7FC00000u) : none ? 0.f : r.rstd * a * (1.f / 127.f);
    r.top = top;
    r.low = low;
    return r;
}

// The code of an element so near to the border between two codes that rounded products do not tell on which side it lies:
// the sign of 254 h w - b a, b twice the border.  Both products are sums of two numbers, p + e and top + low (all of
// them times a power of two where they are tiny or huge), and what is left of 254 p - b top, of e's and of low's
// products are exact sums.
__device__ __noinline__ float exact_code(float h, float w, float b, uint32_t top_bits, uint32_t low_bits)
{
    float top = __uint_as_float(top_bits), low = from_ordered(low_bits);
    if (top < SMALL || top > 1.f / SMALL) {
        const bool first = (fabsf(h) < fabsf(w)) == (top < SMALL);       // whose range bears it
        const float f = top < SMALL ? UP : 1.f / UP;
        h *= first ? f : 1.f;
        w *= first ? 1.f : f;
        if (top > 1.f) low *= f;
        top *= f;
    }
    const float p = h * w, e = __fmaf_rn(h, w, -p);
    const float u = b * top, t = __fsub_rn(__fmaf_rn(254.f, p, -u), __fmaf_rn(b, top, -u));
    const float x = 254.f * e, y = b * low, v = __fsub_rn(x, y), z = __fsub_rn(v, x);
    const float vl = __fsub_rn(__fsub_rn(x, __fsub_rn(v, z)), __fadd_rn(y, z));          // x - y = v + vl
    const float rest = __fadd_rn(vl, __fsub_rn(__fmaf_rn(254.f, e, -x), __fmaf_rn(b, low, -y)));
    const float off = __fadd_rn(__fadd_rn(t, v), rest);
    return 0.5f * b + (off < 0.f ? -0.5f : 0.5f);
}
// Codes floor(127 h w / a + 1/2) of N elements, as MAGIC and the code (whose low byte is the code's).  The rounded product
// times the rounded 127 / a is off by 2^-23 of itself (and 2^-46 of it): times 1 +- 2^-22 it gives the code twice.  Where
// it does not, the element lies next to a border (one in 60000; rows of small integers meet borders often), and its
// code is found exactly.
constexpr float MAGIC = 12582912.f;                            // 1.5 2^23
template <int N> __device__ __forceinline__ void codes_of(const float (&h)[N], const float (&w)[N], const RowQuant &r, float (&t)[N])
{
    if (r.inv == 0.f) {
#pragma unroll
        for (int i = 0; i < N; ++i) t[i] = MAGIC;
        return;
    }
    uint32_t open = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float p = h[i] * w[i];
        t[i] = __fmaf_rn(p, r.inv, MAGIC);
        open |= __float_as_uint(t[i]) ^ __float_as_uint(__fmaf_rn(p, r.up, MAGIC));
    }
    if (!open) return;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float up = __fmaf_rn(h[i] * w[i], r.up, MAGIC);
        if (t[i] != up) t[i] = MAGIC + exact_code(h[i], w[i], __fadd_rn(__fsub_rn(t[i], MAGIC), __fsub_rn(up, MAGIC)), r.top, r.low);
    }
}

// outputs of eight elements at flat index `at`, and of one
template <class T, bool EIGHT>
__device__ __forceinline__ void write_outputs(const FwdParams &p, int64_t at, const float (&h)[8], const float (&w)[8],
                                              const RowQuant &r)
{
    if (p.h) store_vec((T *)p.h + at, h);
    float y[8];
    if constexpr (EIGHT) {
        codes_of<8>(h, w, r, y);
        if (p.codes) store_codes(p.codes + at, y);
        if (!p.y) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = r.s * __fsub_rn(y[i], MAGIC);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = h[i] * r.rstd * w[i];
    }
    if (p.y) store_vec((T *)p.y + at, y);
}
template <class T, bool EIGHT>
__device__ __forceinline__ void write_output(const FwdParams &p, int64_t at, float h, float w, const RowQuant &r)
{
    if (p.h) ((T *)p.h)[at] = dsq_from_f32<T>(h);
    float y = h * r.rstd * w;
    if constexpr (EIGHT) {
        const float h1[1] = {h}, w1[1] = {w};
        float code[1];
        codes_of<1>(h1, w1, r, code);
        y = r.s * __fsub_rn(code[0], MAGIC);
        if (p.codes) p.codes[at] = (int8_t)__float_as_uint(code[0]);
    }
    if (p.y) ((T *)p.y)[at] = dsq_from_f32<T>(y);
}

// single elements of a row a thread takes (14 at most)
template <int TPR, bool ALIGNED> struct Singles { static constexpr int N = ALIGNED ? 0 : TPR >= 16 ? 1 : 2; };

// Blocks an SM that are given registers for: what the usual path needs.  (Left to the compiler the paths of exact codes and of
// rows out of range take more, for rows of one vector a thread: 16384 x 1024 in bf16 to 8 bits 29.3 us, 27.4 with three
// blocks of 256; with four it spills, 29.0.  Of two vectors: 8192 x 4096 47.4 with two blocks, 44.4 with three; rows of 2048, which
// spill then, 25.3 and 36.5.)
__host__ __device__ constexpr int fwd_blocks(int size, int tpr, int items, bool aligned, bool eight)
{
    if (items == 2) return !eight ? 1 : size == 2 && tpr == 256 ? 3 : 512 / block_of(tpr);
    if (tpr >= 512) return (size == 2 || !eight ? 1024 : 512) / block_of(tpr) + (tpr == 1024 && size == 4 && eight);
    return size == 2 && aligned && !eight ? 4 : 3;
}

// TPR threads a row, ITEMS vectors of eight a thread
template <class T, int TPR, int ITEMS, bool ALIGNED, bool EIGHT>
__global__ void __launch_bounds__(block_of(TPR), fwd_blocks(sizeof(T), TPR, ITEMS, ALIGNED, EIGHT)) rmsnorm_fwd_kernel(const FwdParams p)
{
    constexpr int RPB = block_of(TPR) / TPR, ONES = Singles<TPR, ALIGNED>::N, SLOTS = ONES ? ONES : 1;
    __shared__ float4 red[2][block_of(TPR) / 32];
    const int sub = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const int64_t step = (int64_t)gridDim.x * RPB;          // (a multiple of 8 unless ALIGNED)
    const int64_t first = (int64_t)blockIdx.x * RPB + sub;
    const int K = p.K;
    const Cut cut = cut_of<ALIGNED>(first, K);
    const T *x = (const T *)p.x, *res = (const T *)p.res;
    grid_dependency_wait();
    grid_launch_dependents();
    float w[ITEMS][8], w1[SLOTS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) load_weight<ALIGNED>(p.w + cut.head + 8 * (t + i * TPR), t + i * TPR < cut.nv, w[i]);
#pragma unroll
    for (int i = 0; i < ONES; ++i) w1[i] = t + i * TPR < cut.singles ? __ldg(p.w + single_of(cut, t + i * TPR)) : 0.f;

    DsqRaw8<T> xr[ITEMS], rr[ITEMS];
    T x1[SLOTS], r1[SLOTS];           // (as they come: nothing here waits for them)
    auto load = [&](int64_t row) {
        if (row >= p.M) return;
        const int64_t at = row * K + cut.head;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int v = t + i * TPR;
            if (v < cut.nv) {
                xr[i] = dsq_load8(x + at + 8 * v);
                if (res) rr[i] = dsq_load8(res + at + 8 * v);
            }
        }
#pragma unroll
        for (int i = 0; i < ONES; ++i)
            if (t + i * TPR < cut.singles) {
                const int64_t one = row * K + single_of(cut, t + i * TPR);
                x1[i] = x[one];
                if (res) r1[i] = res[one];
            }
    };
    load(first);
    int buf = 0;
    for (int64_t base = (int64_t)blockIdx.x * RPB; base < p.M; base += step, buf ^= 1) {
        const int64_t row = base + sub, at = row * K + cut.head;
        float h[ITEMS][8], one[SLOTS];
        float sum = 0.f, most = 0.f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const bool in = row < p.M && t + i * TPR < cut.nv;
            dsq_unpack8(xr[i], h[i]);
            if (res) {
                float a[8];
                dsq_unpack8(rr[i], a);
#pragma unroll
                for (int k = 0; k < 8; ++k) h[i][k] += a[k];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (!in) h[i][k] = 0.f;
                sum = __fmaf_rn(h[i][k], h[i][k], sum);
            }
            if (EIGHT) most = largest<8>(most, h[i], w[i]);
        }
#pragma unroll
        for (int i = 0; i < ONES; ++i) {
            one[i] = row < p.M && t + i * TPR < cut.singles ? dsq_to_f32(x1[i]) + (res ? dsq_to_f32(r1[i]) : 0.f) : 0.f;
            sum = __fmaf_rn(one[i], one[i], sum);
            if (EIGHT) most = max3(most, most, fabsf(one[i] * w1[i]));
        }
        load(row + step);
        uint32_t top = __float_as_uint(most), low = 0;
        if constexpr (EIGHT) {
            const float own = most;
            most = -INFINITY;
            auto each = [&](auto tiny) {
#pragma unroll
                for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                    for (int k = 0; k < 8; ++k) most = above<decltype(tiny)::value>(most, h[i][k], w[i][k], own);
#pragma unroll
                for (int i = 0; i < ONES; ++i) most = above<decltype(tiny)::value>(most, one[i], w1[i], own);
            };
            if (own >= SMALL || own == 0.f) each(std::false_type());
            else each(std::true_type());
            low = ordered(most);
        }
        const bool far = reduce_row_low<TPR, EIGHT>(sum, top, low, red[buf], p.inv_k, p.eps);
        float rstd = __fdiv_rn(1.f, __fsqrt_rn(__fmaf_rn(sum, p.inv_k, p.eps)));
        if (far) {                // (rows in range beside one that is not keep theirs)
            const float f = far_factor(sum, p.inv_k, p.eps);
            float again = 0.f;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int k = 0; k < 8; ++k) again = __fmaf_rn(h[i][k] * f, h[i][k] * f, again);
#pragma unroll
            for (int i = 0; i < ONES; ++i) again = __fmaf_rn(one[i] * f, one[i] * f, again);
            if (TPR > 32) __syncthreads();                   // red[buf] has been read
            uint32_t none = 0, none2 = 0;
            reduce_row_low<TPR, false>(again, none, none2, red[buf], 1.f, 1.f);
            if (out_of_range(__fmaf_rn(sum, p.inv_k, p.eps))) rstd = far_rstd(again, f, p.inv_k, p.eps);
        }
        const RowQuant r = row_quant(rstd, top, low);
        if (row < p.M) {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const int v = t + i * TPR;
                if (v < cut.nv) write_outputs<T, EIGHT>(p, at + 8 * v, h[i], w[i], r);
            }
#pragma unroll
            for (int i = 0; i < ONES; ++i)
                if (t + i * TPR < cut.singles) write_output<T, EIGHT>(p, row * K + single_of(cut, t + i * TPR), one[i], w1[i], r);
            if (t == 0) {
                if (EIGHT) p.scale[row] = r.s;
                if (p.rstd) p.rstd[row] = r.rstd;
            }
        }
    }
}

// rows too long for the registers of a block: read twice, the second time from the caches
template <class T, bool ALIGNED, bool EIGHT>
__global__ void __launch_bounds__(1024, 2) rmsnorm_fwd_long_kernel(const FwdParams p)
{
    __shared__ float2 red[2][32];
    __shared__ uint32_t lows[2];
    if (EIGHT && threadIdx.x < 2) lows[threadIdx.x] = 0;
    const T *x = (const T *)p.x, *res = (const T *)p.res;
    const int K = p.K;
    grid_dependency_wait();
    grid_launch_dependents();
    int buf = 0;
    for (int64_t row = blockIdx.x; row < p.M; row += gridDim.x, buf ^= 1) {
        const Cut cut = cut_of<ALIGNED>(row, K);
        const int64_t at = row * K + cut.head, one = row * K + single_of(cut, threadIdx.x);
        const bool single = threadIdx.x < cut.singles;
        auto value = [&](int v, float (&h)[8], float (&w)[8]) {
            const DsqRaw8<T> a = dsq_load8(x + at + 8 * v);
            if (res) {
                float b[8];
                dsq_unpack8(dsq_load8(res + at + 8 * v), b);
                dsq_unpack8(a, h);
#pragma unroll
                for (int k = 0; k < 8; ++k) h[k] += b[k];
            } else {
                dsq_unpack8(a, h);
            }
            load_weight<ALIGNED>(p.w + cut.head + 8 * v, true, w);
        };
        float sum = 0.f, most = 0.f, h[8], w[8], h1[1] = {0.f}, w1[1] = {0.f};
        if (single) {
            h1[0] = dsq_to_f32(x[one]);
            if (res) h1[0] += dsq_to_f32(res[one]);
            w1[0] = __ldg(p.w + single_of(cut, threadIdx.x));
            sum = h1[0] * h1[0];
            if (EIGHT) most = largest<1>(most, h1, w1);
        }
        for (int v = threadIdx.x; v < cut.nv; v += 1024) {
            value(v, h, w);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum = __fmaf_rn(h[k], h[k], sum);
            if (EIGHT) most = largest<8>(most, h, w);
        }
        uint32_t top = __float_as_uint(most);
        reduce_row<1024>(sum, top, red[buf]);
        uint32_t low = 0;
        if constexpr (EIGHT) {
            // (by the few threads that hold it, which read their part of the row once more: kept by each thread along with
            // its largest product it takes registers, 2048 x 16384 112 us)
            if (__float_as_uint(most) == top) {
                if (single) low = low_of<1>(h1, w1, most);
                for (int v = threadIdx.x; v < cut.nv; v += 1024) {
                    value(v, h, w);
                    low = max(low, low_of<8>(h, w, most));
                }
                atomicMax(&lows[buf], low);
            }
            __syncthreads();
            low = lows[buf];
            if (threadIdx.x == 0) lows[buf ^ 1] = 0;
        }
        float rstd = __fdiv_rn(1.f, __fsqrt_rn(__fmaf_rn(sum, p.inv_k, p.eps)));
        if (out_of_range(__fmaf_rn(sum, p.inv_k, p.eps))) {
            const float f = far_factor(sum, p.inv_k, p.eps);
            float again = single ? h1[0] * f * (h1[0] * f) : 0.f;
            for (int v = threadIdx.x; v < cut.nv; v += 1024) {
                value(v, h, w);
#pragma unroll
                for (int k = 0; k < 8; ++k) again = __fmaf_rn(h[k] * f, h[k] * f, again);
            }
            __syncthreads();                                 // red[buf] has been read
            uint32_t none = 0;
            reduce_row<1024>(again, none, red[buf]);
            rstd = far_rstd(again, f, p.inv_k, p.eps);
        }
        const RowQuant r = row_quant(rstd, top, low);
        for (int v = threadIdx.x; v < cut.nv; v += 1024) {
            value(v, h, w);
            write_outputs<T, EIGHT>(p, at + 8 * v, h, w, r);
        }
        if (single) write_output<T, EIGHT>(p, one, h1[0], w1[0], r);
        if (threadIdx.x == 0) {
            if (EIGHT) p.scale[row] = r.s;
            if (p.rstd) p.rstd[row] = r.rstd;
        }
    }
}

// (16-bit rows: 64 registers, for 1024 threads an SM: 16384 x 1024 36.8 us, so 27.6; binary32 rows
// would spill: 4096 x 4096 50.8, so 57.8)
template <class T, int TPR, int ITEMS, bool ALIGNED>
__global__ void __launch_bounds__(block_of(TPR), sizeof(T) == 2 ? 1024 / block_of(TPR) : 1) rmsnorm_bwd_kernel(const BwdParams p)
{
    constexpr int RPB = block_of(TPR) / TPR, ONES = Singles<TPR, ALIGNED>::N, SLOTS = ONES ? ONES : 1;
    __shared__ float2 red[2][block_of(TPR) / 32];
    __shared__ float wsum[RPB > 1 || !ALIGNED ? TPR * ITEMS * 8 + 16 : 1];
    const int sub = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const int64_t step = (int64_t)gridDim.x * RPB;          // (a multiple of 8 unless ALIGNED)
    const int64_t first = (int64_t)blockIdx.x * RPB + sub;
    const int K = p.K;
    const Cut cut = cut_of<ALIGNED>(first, K);
    const T *gy = (const T *)p.gy, *gh = (const T *)p.gh, *hh = (const T *)p.h;
    grid_dependency_wait();
    grid_launch_dependents();
    float w[ITEMS][8], gw[ITEMS][8], w1[SLOTS], gw1[SLOTS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        load_weight<ALIGNED>(p.w + cut.head + 8 * (t + i * TPR), t + i * TPR < cut.nv, w[i]);
#pragma unroll
        for (int k = 0; k < 8; ++k) gw[i][k] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < ONES; ++i) {
        w1[i] = t + i * TPR < cut.singles ? __ldg(p.w + single_of(cut, t + i * TPR)) : 0.f;
        gw1[i] = 0.f;
    }

    DsqRaw8<T> yr[ITEMS], hr[ITEMS], gr[ITEMS];
    T y1[SLOTS], h1[SLOTS], a1[SLOTS];
    float rs = 0.f;
    auto load = [&](int64_t row) {
        if (row >= p.M) return;
        const int64_t at = row * K + cut.head;
        rs = p.rstd[row];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int v = t + i * TPR;
            if (v < cut.nv) {
                yr[i] = dsq_load8(gy + at + 8 * v);
                hr[i] = dsq_load8(hh + at + 8 * v);
                if (gh) gr[i] = dsq_load8(gh + at + 8 * v);
            }
        }
#pragma unroll
        for (int i = 0; i < ONES; ++i)
            if (t + i * TPR < cut.singles) {
                const int64_t one = row * K + single_of(cut, t + i * TPR);
                y1[i] = gy[one];
                h1[i] = hh[one];
                if (gh) a1[i] = gh[one];
            }
    };
    load(first);
    int buf = 0;
    for (int64_t base = (int64_t)blockIdx.x * RPB; base < p.M; base += step, buf ^= 1) {
        const int64_t row = base + sub, at = row * K + cut.head;
        const float rstd = rs;
        float g[ITEMS][8], n[ITEMS][8], g1[SLOTS], n1[SLOTS], add1[SLOTS];
        DsqRaw8<T> add[ITEMS];
        float sum = 0.f;
        uint32_t none = 0;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const bool in = row < p.M && t + i * TPR < cut.nv;
            dsq_unpack8(yr[i], g[i]);
            dsq_unpack8(hr[i], n[i]);
            add[i] = gr[i];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                n[i][k] = in ? n[i][k] * rstd : 0.f;
                if (!in) g[i][k] = 0.f;
                gw[i][k] = __fmaf_rn(g[i][k], n[i][k], gw[i][k]);
                g[i][k] *= w[i][k];
                sum = __fmaf_rn(g[i][k], n[i][k], sum);
            }
        }
#pragma unroll
        for (int i = 0; i < ONES; ++i) {
            const bool in = row < p.M && t + i * TPR < cut.singles;
            n1[i] = in ? dsq_to_f32(h1[i]) * rstd : 0.f;
            g1[i] = in ? dsq_to_f32(y1[i]) : 0.f;
            add1[i] = in && gh ? dsq_to_f32(a1[i]) : 0.f;
            gw1[i] = __fmaf_rn(g1[i], n1[i], gw1[i]);
            g1[i] *= w1[i];
            sum = __fmaf_rn(g1[i], n1[i], sum);
        }
        load(row + step);
        reduce_row<TPR>(sum, none, red[buf]);
        const float c = sum * p.inv_k;
        if (row < p.M) {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const int v = t + i * TPR;
                if (v >= cut.nv) continue;
                float o[8], a[8];
                if (gh) dsq_unpack8(add[i], a);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    o[k] = rstd * __fmaf_rn(-n[i][k], c, g[i][k]);
                    if (gh) o[k] += a[k];
                }
                store_vec((T *)p.gx + at + 8 * v, o);
            }
#pragma unroll
            for (int i = 0; i < ONES; ++i)
                if (t + i * TPR < cut.singles) {
                    float o = rstd * __fmaf_rn(-n1[i], c, g1[i]);
                    if (gh) o += add1[i];
                    ((T *)p.gx)[row * K + single_of(cut, t + i * TPR)] = dsq_from_f32<T>(o);
                }
        }
    }
    if (!p.part) return;
    // the block's row of sums: those of its rows' threads in turn
    float *part = p.part + (int64_t)blockIdx.x * K;
    if constexpr (RPB == 1 && ALIGNED) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int col = 8 * (t + i * TPR);
            if (t + i * TPR >= cut.nv) continue;
            reinterpret_cast<float4 *>(part + col)[0] = make_float4(gw[i][0], gw[i][1], gw[i][2], gw[i][3]);
            reinterpret_cast<float4 *>(part + col)[1] = make_float4(gw[i][4], gw[i][5], gw[i][6], gw[i][7]);
        }
    } else {
        for (int s = 0; s < RPB; ++s) {
            if (sub == s) {
#pragma unroll
                for (int i = 0; i < ITEMS; ++i) {
                    const int col = cut.head + 8 * (t + i * TPR);
                    if (t + i * TPR >= cut.nv) continue;
#pragma unroll
                    for (int k = 0; k < 8; ++k) wsum[col + k] = s ? wsum[col + k] + gw[i][k] : gw[i][k];
                }
#pragma unroll
                for (int i = 0; i < ONES; ++i) {
                    const int col = single_of(cut, t + i * TPR);
                    if (t + i * TPR < cut.singles) wsum[col] = s ? wsum[col] + gw1[i] : gw1[i];
                }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < K; c += block_of(TPR)) part[c] = wsum[c];
    }
}

// Long rows: read twice, the sums of grad_w in shared memory, element k of vector v at k nv + v (the
// threads of a warp side by side); a thread's own, since the block's rows are cut alike, being a
// multiple of eight apart.  Two vectors' loads are on their way together.
template <class T, bool ALIGNED>
__global__ void __launch_bounds__(1024) rmsnorm_bwd_long_kernel(const BwdParams p)
{
    extern __shared__ float gw[];
    __shared__ float2 red[2][32];
    const T *gy = (const T *)p.gy, *gh = (const T *)p.gh, *hh = (const T *)p.h;
    const int K = p.K;
    const Cut cut = cut_of<ALIGNED>(blockIdx.x, K);
    const bool single = threadIdx.x < cut.singles;
    for (int c = threadIdx.x; c < 8 * cut.nv; c += 1024) gw[c] = 0.f;
    __syncthreads();
    grid_dependency_wait();
    grid_launch_dependents();
    const float w1 = single ? __ldg(p.w + single_of(cut, threadIdx.x)) : 0.f;
    float gw1 = 0.f;
    int buf = 0;
    for (int64_t row = blockIdx.x; row < p.M; row += gridDim.x, buf ^= 1) {
        const int64_t at = row * K + cut.head, one = row * K + single_of(cut, threadIdx.x);
        const float rstd = p.rstd[row];
        float sum = 0.f, g[8], n[8], w[8], g1 = 0.f, n1 = 0.f;
        uint32_t none = 0;
        if (single) {
            g1 = dsq_to_f32(gy[one]);
            n1 = dsq_to_f32(hh[one]) * rstd;
            gw1 = __fmaf_rn(g1, n1, gw1);
            g1 *= w1;
            sum = g1 * n1;
        }
        for (int v0 = threadIdx.x; v0 < cut.nv; v0 += 2048) {
            DsqRaw8<T> yr[2], hr[2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (v0 + 1024 * i < cut.nv) {
                    yr[i] = dsq_load8(gy + at + 8 * (v0 + 1024 * i));
                    hr[i] = dsq_load8(hh + at + 8 * (v0 + 1024 * i));
                }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int v = v0 + 1024 * i;
                if (v >= cut.nv) break;
                dsq_unpack8(yr[i], g);
                dsq_unpack8(hr[i], n);
                load_weight<ALIGNED>(p.w + cut.head + 8 * v, true, w);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    n[k] *= rstd;
                    gw[k * cut.nv + v] = __fmaf_rn(g[k], n[k], gw[k * cut.nv + v]);
                    sum = __fmaf_rn(g[k] * w[k], n[k], sum);
                }
            }
        }
        reduce_row<1024>(sum, none, red[buf]);
        const float c = sum * p.inv_k;
        for (int v0 = threadIdx.x; v0 < cut.nv; v0 += 2048) {
            DsqRaw8<T> yr[2], hr[2], gr[2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (v0 + 1024 * i < cut.nv) {
                    yr[i] = dsq_load8(gy + at + 8 * (v0 + 1024 * i));
                    hr[i] = dsq_load8(hh + at + 8 * (v0 + 1024 * i));
                    if (gh) gr[i] = dsq_load8(gh + at + 8 * (v0 + 1024 * i));
                }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int v = v0 + 1024 * i;
                if (v >= cut.nv) break;
                dsq_unpack8(yr[i], g);
                dsq_unpack8(hr[i], n);
                load_weight<ALIGNED>(p.w + cut.head + 8 * v, true, w);
                float a[8], o[8];
                if (gh) dsq_unpack8(gr[i], a);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    o[k] = rstd * __fmaf_rn(-(n[k] * rstd), c, g[k] * w[k]);
                    if (gh) o[k] += a[k];
                }
                store_vec((T *)p.gx + at + 8 * v, o);
            }
        }
        if (single) {
            float o = rstd * __fmaf_rn(-n1, c, g1);
            if (gh) o += dsq_to_f32(gh[one]);
            ((T *)p.gx)[one] = dsq_from_f32<T>(o);
        }
    }
    if (!p.part) return;
    __syncthreads();
    float *part = p.part + (int64_t)blockIdx.x * K;
    for (int c = threadIdx.x; c < 8 * cut.nv; c += 1024) part[cut.head + c] = gw[(c & 7) * cut.nv + (c >> 3)];
    if (single) part[single_of(cut, threadIdx.x)] = gw1;
}

// grad_w[k] = sum over the blocks of their sums, in one order: 16 threads a row of sums, 64 rows at a time, eight
// loads of a thread on their way together
constexpr int SUM_ROWS = 64, SUM_COLS = 16;
__global__ void __launch_bounds__(SUM_COLS * SUM_ROWS) weight_sum_kernel(const float *part, int rows, int K, float *out)
{
    __shared__ float s[SUM_ROWS][SUM_COLS + 1];
    const int x = threadIdx.x % SUM_COLS, y = threadIdx.x / SUM_COLS;
    const int col = blockIdx.x * SUM_COLS + x;
    grid_dependency_wait();
    grid_launch_dependents();
    float a = 0.f;
    if (col < K)
        for (int r = y; r < rows; r += 8 * SUM_ROWS) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = r + i * SUM_ROWS < rows ? __ldcg(part + (int64_t)(r + i * SUM_ROWS) * K + col) : 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) a += v[i];
        }
    s[y][x] = a;
    __syncthreads();
    // (a column's sums, over the lanes of a warp)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (warp >= SUM_COLS) return;
    a = 0.f;
#pragma unroll
    for (int i = 0; i < SUM_ROWS / 32; ++i) a += s[lane + 32 * i][warp];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a += __shfl_xor_sync(~0u, a, o);
    if (lane == 0 && blockIdx.x * SUM_COLS + warp < K) out[blockIdx.x * SUM_COLS + warp] = a;
}

// threads a row and vectors a thread, of K elements (eight threads take up to 14 single ones).  0: too
// long for registers
struct Form { int tpr, items; };
Form fwd_form(int64_t K)
{
    const int64_t nv = K / 8;
    if (K % 8 == 0 && nv > 128 && nv <= 1024) return nv <= 256 ? Form{128, 2} : nv <= 512 ? Form{256, 2} : Form{512, 2};
    for (int tpr = 8; tpr <= 1024; tpr *= 2)
        if (nv <= tpr) return {tpr, 1};
    return {0, 0};
}
Form bwd_form(int64_t K)
{
    const int64_t nv = K / 8;
    for (int tpr = 8; tpr <= 1024; tpr *= 2)
        if (nv <= tpr) return {tpr, 1};
    return {0, 0};
}

// Blocks: what is resident together (per_sm: of the kernel; 0: as many as any takes), a multiple of
// eight rows where rows shift; of long rows `rows` a block at least beyond one block an SM: each block
// leaves a row of sums (backward, us, one, two, three and four rows: 1000 x 2048 9.7, 7.7, 8.4, 8.0; 1111 x
// 1777 10.4, 9.9, 9.5, 9.0; 600 x 2000 8.6, 6.4, 6.8, 7.0; 1500 x 1500 10.9, 11.0, 9.2, 10.1; without grad_w
// one is best: 1111 x 1777 4.9, four 5.5).
int grid_of(int64_t M, int64_t K, int tpr, int per_sm, int rows = 1)
{
    const int sms = dsq_sm_count() > 0 ? dsq_sm_count() : 148;
    const int block = tpr ? block_of(tpr) : 1024, rpb = tpr ? block / tpr : 1;
    int64_t g = (M + rpb - 1) / rpb;
    if (rpb == 1 && g > sms) g = (M + rows - 1) / rows > sms ? (M + rows - 1) / rows : sms;
    const int64_t most = (int64_t)sms * (tpr == 0 ? per_sm : per_sm > 0 && per_sm < 1024 / block ? per_sm : 1024 / block);
    if (g > most) g = most;
    if (K % 8 && rpb < 8) {
        const int64_t unit = 8 / rpb;
        // (never more than fit: four blocks of 152 in a second wave took as long as the first 148)
        g = g + unit - 1 > most ? most / unit * unit : (g + unit - 1) / unit * unit;
    }
    return (int)g;
}

template <class K> int blocks_per_sm(K kernel, int block, std::atomic<int> *cached)
{
    int n = cached->load(std::memory_order_relaxed);
    if (n > 0) return n;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, block, 0) != cudaSuccess || n < 1) {
        cudaGetLastError();
        return 0;
    }
    cached->store(n, std::memory_order_relaxed);
    return n;
}

template <class T, bool ALIGNED, bool EIGHT> int fwd_launch(const FwdParams &p, cudaStream_t s)
{
    const Form f = fwd_form(p.K);
    const int pdl = dsq_launch_hooks().pdl;
#define FWD(TPR, ITEMS) \
    if (f.tpr == TPR && f.items == ITEMS) { \
        static std::atomic<int> fit{0}; \
        const auto kernel = rmsnorm_fwd_kernel<T, TPR, ITEMS, ALIGNED, EIGHT>; \
        const dim3 grid(grid_of(p.M, p.K, TPR, blocks_per_sm(kernel, block_of(TPR), &fit))); \
        return dsq_launch(kernel, grid, dim3(block_of(TPR)), 0, s, pdl, 0, p); \
    }
    FWD(8, 1) FWD(16, 1) FWD(32, 1) FWD(64, 1) FWD(128, 1)
    if constexpr (ALIGNED) {
        FWD(128, 2) FWD(256, 2) FWD(512, 2)
    } else {
        FWD(256, 1) FWD(512, 1) FWD(1024, 1)
    }
#undef FWD
    return dsq_launch(rmsnorm_fwd_long_kernel<T, ALIGNED, EIGHT>, dim3(grid_of(p.M, p.K, 0, 2)), dim3(1024), 0, s, pdl, 0, p);
}

template <class T> int fwd_pick(const FwdParams &p, cudaStream_t s)
{
    const bool al = p.K % 8 == 0;
    if (p.scale) return al ? fwd_launch<T, true, true>(p, s) : fwd_launch<T, false, true>(p, s);
    return al ? fwd_launch<T, true, false>(p, s) : fwd_launch<T, false, false>(p, s);
}

// (the workspace is sized for the most blocks that any type takes)
int bwd_grid(int64_t M, int64_t K) { return grid_of(M, K, bwd_form(K).tpr, bwd_form(K).tpr ? 0 : 1); }

template <class T, bool ALIGNED> int bwd_launch(const BwdParams &p, cudaStream_t s, int *blocks)
{
    const Form f = bwd_form(p.K);
    const int pdl = dsq_launch_hooks().pdl;
#define BWD(TPR, ITEMS) \
    if (f.tpr == TPR && f.items == ITEMS) { \
        static std::atomic<int> fit{0}; \
        const auto kernel = rmsnorm_bwd_kernel<T, TPR, ITEMS, ALIGNED>; \
        *blocks = grid_of(p.M, p.K, TPR, blocks_per_sm(kernel, block_of(TPR), &fit), p.part ? 3 : 1); \
        return dsq_launch(kernel, dim3(*blocks), dim3(block_of(TPR)), 0, s, pdl, 0, p); \
    }
    BWD(8, 1) BWD(16, 1) BWD(32, 1) BWD(64, 1) BWD(128, 1) BWD(256, 1) BWD(512, 1) BWD(1024, 1)
#undef BWD
    static std::atomic<unsigned long long> configured{0};
    const int st = dsq_allow_smem((const void *)rmsnorm_bwd_long_kernel<T, ALIGNED>, (int)(MAX_K * 4), &configured);
    if (st) return st;
    *blocks = grid_of(p.M, p.K, 0, 1);
    return dsq_launch(rmsnorm_bwd_long_kernel<T, ALIGNED>, dim3(*blocks), dim3(1024), (size_t)p.K * 4, s, pdl, 0, p);
}

int check_shape(int64_t M, int64_t K, int dtype)
{
    if (!dsq_is_float_type(dtype)) return DSQ_ERR_UNSUPPORTED;
    if (M <= 0 || K <= 0) return DSQ_ERR_SHAPE;
    if (K > MAX_K || M > (int64_t)1 << 40) return DSQ_ERR_SIZE;
    return DSQ_OK;
}

}  // namespace

extern "C" {

int dsq_rmsnorm_fwd(const void *x, const void *residual, const float *weight, int64_t M, int64_t K,
                    int dtype, float eps, void *h_out, void *y_out, int8_t *codes_out,
                    float *scale_out, float *rstd_out, void *stream)
{
    if (!x || !weight || (!y_out && !codes_out) || (codes_out && !scale_out)) return DSQ_ERR_NULL;
    const int st = check_shape(M, K, dtype);
    if (st) return st;
    if (!dsq_finite(eps) || eps < 0.f) return DSQ_ERR_RANGE;
    const void *all[] = {x, residual, weight, h_out, y_out, codes_out, scale_out, rstd_out};
    for (const void *a : all)
        if (!dsq_aligned16(a)) return DSQ_ERR_ALIGN;
    FwdParams p;
    p.x = x; p.res = residual; p.w = weight;
    p.h = h_out; p.y = y_out; p.codes = codes_out; p.scale = scale_out; p.rstd = rstd_out;
    p.M = M; p.K = (int)K;
    p.eps = eps; p.inv_k = (float)(1.0 / (double)K);
    cudaStream_t s = (cudaStream_t)stream;
    switch (dtype) {
    case DSQ_F32: return fwd_pick<float>(p, s);
    case DSQ_BF16: return fwd_pick<__nv_bfloat16>(p, s);
    default: return fwd_pick<__half>(p, s);
    }
}

size_t dsq_rmsnorm_bwd_workspace_bytes(int64_t M, int64_t K)
{
    if (M <= 0 || K <= 0 || K > MAX_K) return DSQ_WS_BYTES;
    return DSQ_WS_BYTES + (size_t)bwd_grid(M, K) * (size_t)K * 4;
}

int dsq_rmsnorm_bwd(const void *grad_y, const void *grad_h, const void *h, const float *weight,
                    const float *rstd, int64_t M, int64_t K, int dtype, void *grad_x,
                    float *grad_weight, void *workspace, size_t ws_bytes, void *stream)
{
    if (!grad_y || !h || !weight || !rstd || !grad_x || (grad_weight && !workspace)) return DSQ_ERR_NULL;
    int st = check_shape(M, K, dtype);
    if (st) return st;
    const void *all[] = {grad_y, grad_h, h, weight, rstd, grad_x, grad_weight, workspace};
    for (const void *a : all)
        if (!dsq_aligned16(a)) return DSQ_ERR_ALIGN;
    if (grad_weight && ws_bytes < dsq_rmsnorm_bwd_workspace_bytes(M, K)) return DSQ_ERR_SIZE;
    BwdParams p;
    p.gy = grad_y; p.gh = grad_h; p.h = h; p.w = weight; p.rstd = rstd; p.gx = grad_x;
    p.part = grad_weight ? (float *)((char *)workspace + DSQ_WS_BYTES) : nullptr;
    p.M = M; p.K = (int)K;
    p.inv_k = (float)(1.0 / (double)K);
    cudaStream_t s = (cudaStream_t)stream;
    const bool al = K % 8 == 0;
    int blocks = 0;
    switch (dtype) {
    case DSQ_F32: st = al ? bwd_launch<float, true>(p, s, &blocks) : bwd_launch<float, false>(p, s, &blocks); break;
    case DSQ_BF16: st = al ? bwd_launch<__nv_bfloat16, true>(p, s, &blocks) : bwd_launch<__nv_bfloat16, false>(p, s, &blocks); break;
    default: st = al ? bwd_launch<__half, true>(p, s, &blocks) : bwd_launch<__half, false>(p, s, &blocks); break;
    }
    if (st || !grad_weight) return st;
    return dsq_launch(weight_sum_kernel, dim3((unsigned)((K + SUM_COLS - 1) / SUM_COLS)), dim3(SUM_COLS * SUM_ROWS), 0, s,
                      dsq_launch_hooks().pdl, 0, p.part, blocks, (int)K, grad_weight);
}

}  // extern "C"
