// 4-bit weights with a scale per group of consecutive weights of a row (paper Eq. 2,
// Algorithm 1 steps 1, 3, 4 on weights, the clip range [-a, a] taken from each
// group's largest magnitude a), and the values such codes stand for.
//
//   q = floor((w + a) 15 / (2 a) + 1/2) = floor(15 w / (2 a) + 8),  c = q - 8,
//   scale = a / 15,  w^ = scale (2 c + 1)
//
// The code is exact: weights kept in 16 bits lie on the border between two codes
// often (w / a a ratio of small integers), and which side a rounded reciprocal puts
// them on is chance.  The border nearest to the estimate, w = a (2 b - 16) / 15, is
// compared with w itself: p = a m and its rounding error e (m = 2 b - 16, an even
// integer of at most 16 in magnitude) hold a m exactly, and fma(15, w, -p) - e has the
// sign of 15 w - a m.
//
// Bound: memory (bf16 in 2.5 bytes a weight, values out 2.5).
#include "dsq_groups.h"
#include "dsq_ptx.cuh"
#include "dsq_types.cuh"

using dsq_ptx::grid_dependency_wait;
using dsq_ptx::grid_launch_dependents;

namespace {

struct QuantParams {
    const void *w;
    uint32_t *codes;
    float *scales;            // [groups][N]
    int64_t N;
    int K, pw;                // pw: 32-bit words of a row (8 codes each)
    int group_words;          // words of a group
    int row_words;            // words of a row in whole groups
};

// What a group's codes are made with: everything scaled by a power of two that brings a
// to [1, 2) (smaller for the last subnormal bits, up to 4 at the top of the range), so that
// nothing below over- or underflows.
struct Range { float f, a, inv, scale; bool bad; };
__device__ __forceinline__ Range range_of(uint32_t top)
{
    Range r;
    const float a = __uint_as_float(top);
    r.bad = top >= 0x7F800000u;                               // an infinity or a NaN in the group
    const int e = min(max((int)(top >> 23) - 127, -126), 126);
    r.f = __uint_as_float((uint32_t)(127 - e) << 23);
    r.a = a * r.f;
    r.inv = r.bad || a == 0.f ? 0.f : __fdiv_rn(7.5f, r.a);
    r.scale = r.bad ? __uint_as_float(0x7FC00000u) : __fdiv_rn(a, 15.f);
    return r;
}
// four bits of the signed code (of a group of zeros: 0; of one that is not finite: -8)
__device__ __forceinline__ uint32_t code_of(float w, const Range &r)
{
    if (r.bad) return 8u;
    const float x = w * r.f;
    const float b = rintf(__fmaf_rn(x, r.inv, 8.f));
    const float m = __fmaf_rn(2.f, b, -16.f);
    const float p = __fmul_rn(r.a, m), e = __fmaf_rn(r.a, m, -p);
    const float d = m == 0.f ? w : __fsub_rn(__fmaf_rn(15.f, x, -p), e);
    const int q = (int)b - (d >= 0.f ? 0 : 1);
    return (uint32_t)min(max(q, 0), 15) ^ 8u;
}

// eight weights from column k of a row; those behind the row's end are 0
template <class T, bool VEC>
__device__ __forceinline__ void load_weights(const T *w, int64_t row, int k, int K, float (&f)[8])
{
    if (VEC) {
        if (k < K) {
            dsq_unpack8(dsq_load8(w + row * K + k), f);
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = 0.f;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = k + i < K ? dsq_to_f32(w[row * K + k + i]) : 0.f;
    }
}
__device__ __forceinline__ uint32_t top_of(const float (&f)[8])
{
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) t = max(t, __float_as_uint(f[i]) & 0x7FFFFFFFu);
    return t;
}
__device__ __forceinline__ uint32_t word_of(const float (&f)[8], int k, int K, const Range &r)
{
    uint32_t v = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) v |= (k + i < K ? code_of(f[i], r) : 0u) << (4 * i);
    return v;
}

// Groups of 32, 64, 128 or 256: 4 to 32 neighbouring threads hold one, a word of codes
// each (a row's last group, cut short, has idle threads: groups start at lanes that are
// multiples of their size).
constexpr int UNROLL = 2;
template <class T, bool VEC>
__global__ void __launch_bounds__(256) quantize_words_kernel(const QuantParams p)
{
    grid_dependency_wait();
    const int64_t base = (int64_t)blockIdx.x * (256 * UNROLL);
    const int64_t row0 = base / p.row_words;
    const unsigned rest = (unsigned)(base - row0 * p.row_words) + threadIdx.x;
    float f[UNROLL][8];
    int64_t row[UNROLL];
    int word[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const unsigned i = rest + 256 * u, r = i / (unsigned)p.row_words;
        row[u] = row0 + r;
        word[u] = (int)(i - r * (unsigned)p.row_words);
        load_weights<T, VEC>((const T *)p.w, row[u], row[u] < p.N ? 8 * word[u] : p.K, p.K, f[u]);
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        uint32_t top = top_of(f[u]);
        for (int o = 1; o < p.group_words; o <<= 1) top = max(top, __shfl_xor_sync(~0u, top, o));
        if (row[u] >= p.N || word[u] >= p.pw) continue;
        const Range r = range_of(top);
        p.codes[row[u] * p.pw + word[u]] = word_of(f[u], 8 * word[u], p.K, r);
        const int g = word[u] / p.group_words;
        if (word[u] == g * p.group_words) p.scales[g * p.N + row[u]] = r.scale;
    }
}

// Any other multiple of 32: a warp a group, its weights read twice (the second time from
// the caches).
template <class T, bool VEC>
__global__ void __launch_bounds__(256) quantize_group_kernel(const QuantParams p, int groups)
{
    grid_dependency_wait();
    const int lane = threadIdx.x & 31;
    const int64_t at = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int64_t row = at / groups;
    if (row >= p.N) return;
    const int g = (int)(at - row * groups);
    const int w0 = g * p.group_words, w1 = min(w0 + p.group_words, p.pw);
    float f[8];
    uint32_t top = 0;
    for (int w = w0 + lane; w < w1; w += 32) {
        load_weights<T, VEC>((const T *)p.w, row, 8 * w, p.K, f);
        top = max(top, top_of(f));
    }
    const Range r = range_of(__reduce_max_sync(~0u, top));
    for (int w = w0 + lane; w < w1; w += 32) {
        load_weights<T, VEC>((const T *)p.w, row, 8 * w, p.K, f);
        p.codes[row * p.pw + w] = word_of(f, 8 * w, p.K, r);
    }
    if (lane == 0) p.scales[g * p.N + row] = r.scale;
}

struct ValueParams {
    const uint32_t *codes;
    const float *scales;
    void *out;
    int64_t N;
    int K, pw, group_words;
    int odd;                  // values 2 c + 1 (else c)
};

// A thread a word of eight codes: reads and writes of a warp are contiguous.
template <class T, bool VEC>
__global__ void __launch_bounds__(256) dequantize_kernel(const ValueParams p)
{
    grid_dependency_wait();
    grid_launch_dependents();
    const int64_t base = (int64_t)blockIdx.x * (256 * UNROLL);
    const int64_t row0 = base / p.pw;
    const unsigned rest = (unsigned)(base - row0 * p.pw) + threadIdx.x;
    T *out = (T *)p.out;
    uint32_t v[UNROLL];
    float s[UNROLL];
    int64_t row[UNROLL];
    int word[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const unsigned i = rest + 256 * u, r = i / (unsigned)p.pw;
        row[u] = row0 + r;
        word[u] = (int)(i - r * (unsigned)p.pw);
        if (row[u] < p.N && 8 * word[u] < p.K) {
            v[u] = __ldg(p.codes + row[u] * p.pw + word[u]);
            s[u] = __ldg(p.scales + (int64_t)(word[u] / p.group_words) * p.N + row[u]);
        }
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const int k = 8 * word[u];
        if (row[u] >= p.N || k >= p.K) continue;
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = (int)(v[u] << (28 - 4 * i)) >> 28;
            f[i] = s[u] * (float)(p.odd ? 2 * c + 1 : c);
        }
        if (VEC) {
            DsqRaw8<T> r;
            dsq_pack8(f, r);
            dsq_store8(out + row[u] * p.K + k, r);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < p.K) out[row[u] * p.K + k + i] = dsq_from_f32<T>(f[i]);
        }
    }
}

int blocks_of(int64_t words, int per_block, dim3 *grid)
{
    const int64_t g = (words + per_block - 1) / per_block;
    if (g > 0x7FFFFFFF) return DSQ_ERR_SIZE;
    *grid = dim3((unsigned)g);
    return DSQ_OK;
}

template <class T, bool VEC> int quantize(const QuantParams &p, int groups, cudaStream_t s)
{
    dim3 grid;
    const bool words = p.group_words <= 32 && (p.group_words & (p.group_words - 1)) == 0;
    const int st = words ? blocks_of(p.N * p.row_words, 256 * UNROLL, &grid) : blocks_of(p.N * groups, 8, &grid);
    if (st) return st;
    // (what these kernels write are a layer's constants: what follows starts behind them)
    if (words)
        return dsq_launch(quantize_words_kernel<T, VEC>, grid, dim3(256), 0, s, dsq_launch_hooks().pdl, 0, p);
    return dsq_launch(quantize_group_kernel<T, VEC>, grid, dim3(256), 0, s, dsq_launch_hooks().pdl, 0, p, groups);
}

template <class T, bool VEC> int dequantize(const ValueParams &p, cudaStream_t s)
{
    dim3 grid;
    const int st = blocks_of(p.N * p.pw, 256 * UNROLL, &grid);
    if (st) return st;
    return dsq_launch(dequantize_kernel<T, VEC>, grid, dim3(256), 0, s, dsq_launch_hooks().pdl, 0, p);
}

}  // namespace

int dsq_check_groups(int64_t N, int64_t K, int bits, int64_t group)
{
    if (bits < 1 || bits > 4) return DSQ_ERR_BITS;
    if (bits != 4) return DSQ_ERR_UNSUPPORTED;
    if (N <= 0 || K <= 0 || group <= 0) return DSQ_ERR_SHAPE;
    if (group % 32 != 0) return DSQ_ERR_UNSUPPORTED;
    if (K > DSQ_GROUPS_MAX_K || N > (1 << 28)) return DSQ_ERR_SIZE;
    return DSQ_OK;
}

extern "C" {

int64_t dsq_group_count(int64_t K, int64_t group)
{
    return K <= 0 || group <= 0 ? 0 : (K - 1) / group + 1;
}

int dsq_quantize_groups(const void *w, int64_t N, int64_t K, int dtype, int bits, int64_t group,
                        void *codes_out, size_t bytes, float *scales_out, void *stream)
{
    if (!w || !codes_out || !scales_out) return DSQ_ERR_NULL;
    const int st = dsq_check_groups(N, K, bits, group);
    if (st) return st;
    if (!dsq_is_float_type(dtype)) return DSQ_ERR_UNSUPPORTED;
    if (!dsq_aligned16(w) || !dsq_aligned16(codes_out) || !dsq_aligned16(scales_out)) return DSQ_ERR_ALIGN;
    if (bytes < dsq_packed_bytes(N, K, bits)) return DSQ_ERR_SIZE;
    const int groups = (int)dsq_group_count(K, group);
    QuantParams p;
    p.w = w;
    p.codes = (uint32_t *)codes_out;
    p.scales = scales_out;
    p.N = N;
    p.K = (int)K;
    p.pw = (int)(dsq_row_pitch(K, bits) / 4);
    // (a group longer than the row is the row)
    p.group_words = groups == 1 && group > 256 ? p.pw : (int)(group / 8);
    p.row_words = groups * p.group_words;
    cudaStream_t s = (cudaStream_t)stream;
    const bool vec = K % 8 == 0;
    switch (dtype) {
    case DSQ_F32: return vec ? quantize<float, true>(p, groups, s) : quantize<float, false>(p, groups, s);
    case DSQ_BF16: return vec ? quantize<__nv_bfloat16, true>(p, groups, s) : quantize<__nv_bfloat16, false>(p, groups, s);
    default: return vec ? quantize<__half, true>(p, groups, s) : quantize<__half, false>(p, groups, s);
    }
}

int dsq_dequantize_groups(const void *codes, const float *scales, int64_t N, int64_t K, int bits,
                          int64_t group, float w_offset, int dtype, void *values_out, void *stream)
{
    if (!codes || !scales || !values_out) return DSQ_ERR_NULL;
    const int st = dsq_check_groups(N, K, bits, group);
    if (st) return st;
    if (!dsq_finite(w_offset)) return DSQ_ERR_RANGE;
    if (!dsq_is_float_type(dtype) || (w_offset != 0.0f && w_offset != 0.5f)) return DSQ_ERR_UNSUPPORTED;
    if (!dsq_aligned16(codes) || !dsq_aligned16(scales) || !dsq_aligned16(values_out)) return DSQ_ERR_ALIGN;
    ValueParams p;
    p.codes = (const uint32_t *)codes;
    p.scales = scales;
    p.out = values_out;
    p.N = N;
    p.K = (int)K;
    p.pw = (int)(dsq_row_pitch(K, bits) / 4);
    p.group_words = dsq_group_count(K, group) == 1 ? p.pw : (int)(group / 8);
    p.odd = w_offset == 0.5f;
    cudaStream_t s = (cudaStream_t)stream;
    const bool vec = K % 8 == 0;
    switch (dtype) {
    case DSQ_F32: return vec ? dequantize<float, true>(p, s) : dequantize<float, false>(p, s);
    case DSQ_BF16: return vec ? dequantize<__nv_bfloat16, true>(p, s) : dequantize<__nv_bfloat16, false>(p, s);
    default: return vec ? dequantize<__half, true>(p, s) : dequantize<__half, false>(p, s);
    }
}

}  // extern "C"
