// 4-bit weights with a scale per group of consecutive weights of a row (paper Eq. 2,
// Algorithm 1 steps 1, 3, 4 on weights, the clip range [-a, a] taken from each
// group's largest magnitude a), and the values such codes stand for.
//
//   q = floor((w + a) 15 / (2 a) + 1/2) = floor(15 w / (2 a) + 8),  c = q - 8,
//   scale = a / 15,  w^ = scale (2 c + 1)
//
// The code is exact: weights kept in 16 bits lie on the border between two codes
// often (w / a a ratio of small integers), and which side a rounded reciprocal puts
// them on is chance.  c = floor(v), v = 7.5 w / a:
//   * 16-bit weights: a v that is no whole number is 2^-15 away from one at least, where it
//     is above 1 (15 w and 2 a are integers of 15 and 12 bits on one grid, at most three
//     powers of two apart), and 7.5 / a in binary32 is off by 2^-21 of itself: v (1 +- 2^-19),
//     upwards, lies on the right side, and its floor is the code.  Both signs' v are made and rounded
//     down to a whole number in one fused operation each, and the larger one is the upper one;
//   * binary32 weights: with j = rint(v) as far as binary32 gives it, the code is j or j - 1
//     by the sign of 7.5 w - a j, in which the rounding error of a j is taken off.
//
// Bound: memory (bf16 in 2.5 bytes a weight, values out 2.5), with arithmetic close behind (16384 x
// 4096 in groups of 128: codes 31 us, values 30, at the copy's rate 26): the conversions between integers and floating point run at an eighth of the other operations' rate,
// so j is read off the sum with 1.5 2^23, and codes become numbers in the mantissa of 2^23.  A
// thread's column is the same in all its rows, so that nothing is divided per word.
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
    int groups, group_words;  // group_words: words of a group
    int lanes_log;            // 2^lanes_log threads hold a group
    int bx_log;               // 2^bx_log threads of a block along a row
};

// What a group's codes are made with.  Tiny groups are scaled up (exactly), and the comparison
// with a border is a sixteenth of it, so that nothing over- or underflows.
struct Range { float f, a, inv, up, down, scale; bool bad; };      // up, down: inv (1 +- 2^-19)
__device__ __forceinline__ Range range_of(uint32_t top)
{
    Range r;
    const float a = __uint_as_float(top);
    r.bad = top >= 0x7F800000u;                               // an infinity or a NaN in the group
    r.f = a < 7.8886e-31f ? 1.2676506e30f : 1.f;              // below 2^-100: times 2^100
    const float x = a * r.f;
    r.a = x * 0.0625f;
    // (off by its last bits: what is made of it allows for that; finite for a = 0)
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.inv) : "f"(fmaxf(r.a, 1e-37f)));
    r.inv *= 0.46875f;
    r.up = r.inv * (1.f + 1.9073486e-6f);
    r.down = r.inv * (1.f - 1.9073486e-6f);
    // a / 15, rounded once: a quotient, corrected by what is left of a (a division in every
    // thread took 9 us of 67 at 16384 x 4096 in groups of 128)
    constexpr float R15 = 1.f / 15.f;
    const float s = a * R15;
    r.scale = r.bad ? __uint_as_float(0x7FC00000u) : __fmaf_rn(__fmaf_rn(-15.f, s, a), R15, s);
    return r;
}
constexpr float MAGIC = 12582912.f;                           // 1.5 2^23
constexpr uint32_t MAGIC_BITS = 0x4B400000u;
// bits of MAGIC + c, c the signed code (the ends of the range need no clip: |v| <= 7.5)
template <bool WIDE> __device__ __forceinline__ uint32_t code_bits(float x, const Range &r)
{
    if constexpr (WIDE) {
        const float t = __fmaf_rn(x, r.inv, MAGIC);
        const float nj = __fsub_rn(MAGIC, t);                 // -j (never -0)
        const float p = __fmul_rn(r.a, nj);
        // (7.5 x - a j) / 16, rounded down: that of the smallest negative x stays below 0
        const float d = __fadd_rn(__fmaf_rd(0.46875f, x, p), __fmaf_rn(r.a, nj, -p));
        return __float_as_uint(t) + (uint32_t)((int)__float_as_uint(d) >> 31);
    } else {
        return __float_as_uint(fmaxf(__fmaf_rd(x, r.up, MAGIC), __fmaf_rd(x, r.down, MAGIC)));
    }
}

// eight weights from column k of the row at w; those behind its end are 0
template <class T, bool VEC>
__device__ __forceinline__ DsqRaw8<T> load_weights(const T *w, int k, int K)
{
    DsqRaw8<T> r;
    if (VEC) {
        if (k < K) return dsq_load8(w + k);
#pragma unroll
        for (int i = 0; i < (int)(sizeof(r) / 16); ++i) r.v[i] = make_uint4(0u, 0u, 0u, 0u);
    } else {
        // (its own eight, one by one: 4096 x 4100 in bf16 21.4 us; neighbours' through shared memory 26.4)
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = k + i < K ? dsq_to_f32(w[k + i]) : 0.f;
        dsq_pack8(f, r);
    }
    return r;
}
// the largest magnitude's bits, in the type's own bits (those of a NaN are above infinity's)
template <class T> __device__ __forceinline__ uint32_t top_of(const DsqRaw8<T> &r)
{
    if constexpr (sizeof(T) == 2) {
        constexpr uint32_t ABS = 0x7FFF7FFFu;
        const uint32_t t = __vmaxu2(__vmaxu2(r.v[0].x & ABS, r.v[0].y & ABS), __vmaxu2(r.v[0].z & ABS, r.v[0].w & ABS));
        return max(t & 0xFFFFu, t >> 16);
    } else {
        constexpr uint32_t ABS = 0x7FFFFFFFu;
        const uint4 a = r.v[0], b = r.v[1];
        return max(max(max(a.x & ABS, a.y & ABS), max(a.z & ABS, a.w & ABS)),
                   max(max(b.x & ABS, b.y & ABS), max(b.z & ABS, b.w & ABS)));
    }
}
// such bits as binary32's
__device__ __forceinline__ uint32_t wide_bits(uint32_t top, float) { return top; }
__device__ __forceinline__ uint32_t wide_bits(uint32_t top, __nv_bfloat16) { return top << 16; }
__device__ __forceinline__ uint32_t wide_bits(uint32_t top, __half)
{
    return __float_as_uint(__half2float(__ushort_as_half((unsigned short)top))) & 0x7FFFFFFFu;
}
// the word of eight codes; those behind the row's end are 0
template <class T> __device__ __forceinline__ uint32_t word_of(const DsqRaw8<T> &raw, int k, int K, const Range &r)
{
    float f[8];
    dsq_unpack8(raw, f);
    if (r.f != 1.f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] *= r.f;
    }
    uint32_t v = 0;
#pragma unroll
    for (int i = 7; i >= 0; --i) v = v * 16u + code_bits<sizeof(T) == 4>(f[i], r);
    // every term stands for MAGIC_BITS + c: codes made positive, summed without carries, and
    // turned into two's complement nibbles
    constexpr uint32_t ALL = 0x11111111u;
    v = (v - MAGIC_BITS * ALL + 8u * ALL) ^ 0x88888888u;
    if (r.bad) v = 0x88888888u;
    if (k + 8 > K) v = k >= K ? 0u : v & (0xFFFFFFFFu >> (4 * (8 - (K - k))));
    return v;
}

// 2^lanes_log neighbouring threads hold a group, up to WORDS words of codes each (0: any number,
// read twice, the second time from the caches); a thread does ROWS rows.
template <class T, bool VEC, int WORDS, int ROWS>
__global__ void __launch_bounds__(256) quantize_kernel(const QuantParams p)
{
    const int lanes = 1 << p.lanes_log, tx = threadIdx.x & ((1 << p.bx_log) - 1), ty = threadIdx.x >> p.bx_log;
    const int slot = (blockIdx.y << p.bx_log) + tx;
    const int g = slot >> p.lanes_log, l = slot & (lanes - 1);
    const int w0 = g * p.group_words + l, w1 = min((g + 1) * p.group_words, p.pw);
    const int by = 256 >> p.bx_log;
    const int64_t row0 = (int64_t)blockIdx.x * (by * ROWS) + ty;
    const bool in = g < p.groups;
    const T *w = (const T *)p.w;
    grid_dependency_wait();
    if constexpr (WORDS > 0) {
        const int left = (int)min(p.N - row0, (int64_t)ROWS * by);       // rows from row0 on
        DsqRaw8<T> f[ROWS][WORDS];
        uint32_t top[ROWS];
        const T *src = w + row0 * p.K;
#pragma unroll
        for (int u = 0; u < ROWS; ++u, src += (int64_t)by * p.K)
#pragma unroll
            for (int i = 0; i < WORDS; ++i) {
                const int word = w0 + i * lanes;
                f[u][i] = load_weights<T, VEC>(src, in && u * by < left && word < w1 ? 8 * word : p.K, p.K);
            }
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            top[u] = top_of(f[u][0]);
#pragma unroll
            for (int i = 1; i < WORDS; ++i) top[u] = max(top[u], top_of(f[u][i]));
        }
        if constexpr (sizeof(T) == 2 && ROWS % 2 == 0) {                 // two rows' in a register
#pragma unroll
            for (int u = 0; u < ROWS; u += 2) top[u] |= top[u + 1] << 16;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                if (o >= lanes) break;
#pragma unroll
                for (int u = 0; u < ROWS; u += 2) top[u] = __vmaxu2(top[u], __shfl_xor_sync(~0u, top[u], o));
            }
#pragma unroll
            for (int u = 0; u < ROWS; u += 2) {
                top[u + 1] = top[u] >> 16;
                top[u] &= 0xFFFFu;
            }
        } else {
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                if (o >= lanes) break;
#pragma unroll
                for (int u = 0; u < ROWS; ++u) top[u] = max(top[u], __shfl_xor_sync(~0u, top[u], o));
            }
        }
        uint32_t *dst = p.codes + row0 * p.pw;
        float *scale = p.scales + (int64_t)g * p.N + row0;
#pragma unroll
        for (int u = 0; u < ROWS; ++u, dst += (int64_t)by * p.pw, scale += by) {
            if (!in || u * by >= left) continue;
            const Range r = range_of(wide_bits(top[u], T()));
#pragma unroll
            for (int i = 0; i < WORDS; ++i) {
                const int word = w0 + i * lanes;
                if (word < w1) dst[word] = word_of<T>(f[u][i], 8 * word, p.K, r);
            }
            if (l == 0) *scale = r.scale;
        }
    } else {
        const int64_t row = row0;
        const T *src = w + row * p.K;
        uint32_t top = 0;
        const int end = in && row < p.N ? w1 : 0;
        for (int word = w0; word < end; word += lanes)
            top = max(top, top_of(load_weights<T, VEC>(src, 8 * word, p.K)));
        for (int o = 1; o < lanes; o <<= 1) top = max(top, __shfl_xor_sync(~0u, top, o));
        const Range r = range_of(wide_bits(top, T()));
        for (int word = w0; word < end; word += lanes)
            p.codes[row * p.pw + word] = word_of<T>(load_weights<T, VEC>(src, 8 * word, p.K), 8 * word, p.K, r);
        if (l == 0 && end) p.scales[g * p.N + row] = r.scale;
    }
}

struct ValueParams {
    const uint32_t *codes;
    const float *scales;
    void *out;
    int64_t N;
    int K, pw, group_words;
    int odd;                  // values 2 c + 1 (else c)
    int bx_log;
};

// A thread a word of eight codes: reads and writes of a warp are contiguous.
constexpr int VALUE_ROWS = 4;
template <class T, bool VEC>
__global__ void __launch_bounds__(256) dequantize_kernel(const ValueParams p)
{
    const int tx = threadIdx.x & ((1 << p.bx_log) - 1), ty = threadIdx.x >> p.bx_log, by = 256 >> p.bx_log;
    const int word = (blockIdx.y << p.bx_log) + tx, k = 8 * word;
    const int64_t row0 = (int64_t)blockIdx.x * (by * VALUE_ROWS) + ty;
    const float *scales = p.scales + (int64_t)(word / p.group_words) * p.N + row0;
    const int left = (int)min(p.N - row0, (int64_t)VALUE_ROWS * by);     // rows from row0 on
    grid_dependency_wait();
    grid_launch_dependents();
    uint32_t v[VALUE_ROWS];
    float s[VALUE_ROWS];
    const uint32_t *src = p.codes + row0 * p.pw + word;
#pragma unroll
    for (int u = 0; u < VALUE_ROWS; ++u, src += (int64_t)by * p.pw)
        if (u * by < left && k < p.K) {
            v[u] = __ldg(src);
            s[u] = __ldg(scales + u * by);
        }
    // a nibble at bits 1 to 4 of the mantissa of 2^23: with bit 0, 2^23 + 2 q + 1; else 2^23 + 2 q
    // (q = c + 8)
    const uint32_t bits = p.odd ? 0x4B000011u : 0x4B000010u;
    const float half = p.odd ? 1.f : 0.5f;
    T *out = (T *)p.out + row0 * p.K + k;
    __shared__ DsqRaw8<T> turn[VEC ? 1 : 256];
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int u = 0; u < VALUE_ROWS; ++u, out += (int64_t)by * p.K) {
        if (u * by >= left || (VEC && k >= p.K)) continue;               // (of a warp all, where rows are not aligned)
        DsqRaw8<T> r = {};
        if (k < p.K) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t y = i ? v[u] >> (4 * i - 1) : v[u] << 1;
                f[i] = s[u] * ((__uint_as_float((y & 0x1Eu) ^ bits) - 8388624.f) * half);
            }
            dsq_pack8(f, r);
        }
        if (VEC) {
            dsq_store8(out, r);
        } else {
            // through shared memory, to be written element beside element: 1111 x 1777 in binary32 took 9.7 us
            // with a thread's eight written by itself
            __syncwarp();
            turn[threadIdx.x] = r;
            __syncwarp();
            const T *of = reinterpret_cast<const T *>(&turn[threadIdx.x - lane]);
            const int k0 = k - 8 * lane;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k0 + lane + 32 * i < p.K) out[lane + 32 * i - 8 * lane] = of[lane + 32 * i];
        }
    }
}

// A block's threads along a row (a power of two, 32 at least), the rest of them rows; rows along x.
int block_shape(int64_t N, int64_t across, int rows, int *bx_log, dim3 *grid)
{
    int log = 5;
    while (log < 8 && (1 << log) < across) ++log;
    *bx_log = log;
    const int64_t per = (int64_t)(256 >> log) * rows, gx = (N + per - 1) / per;
    const int64_t gy = (across + (1 << log) - 1) >> log;
    if (gx > 0x7FFFFFFF || gy > 65535) return DSQ_ERR_SIZE;
    *grid = dim3((unsigned)gx, (unsigned)gy);
    return DSQ_OK;
}

template <class T, bool VEC> int quantize(QuantParams p, cudaStream_t s)
{
    // Words of a thread: with more of them a group's magnitude and reciprocal are fewer threads' work, with
    // fewer lanes a warp's accesses are shorter pieces.  16384 x 4096 in bf16, us, one, two and four words: groups
    // of 128 43.0, 36.7, 34.0; of 64 42.6, 36.8, 38.7; of 32 42.6, 38.0, 43.7.  4096 x 4096 in binary32, of 64:
    // 16.8, 14.9, 16.6.  Rows that are not aligned, 4096 x 4100 in bf16, of 128: one 21.4, four 27.4.
    const int most = !VEC ? 1 : sizeof(T) == 2 && p.group_words >= 16 ? 4 : 2;
    p.lanes_log = 0;
    while (p.lanes_log < 5 && (most << p.lanes_log) < p.group_words) ++p.lanes_log;
    const int words = (p.group_words + (1 << p.lanes_log) - 1) >> p.lanes_log;      // of a thread
    dim3 grid;
    const int st = block_shape(p.N, (int64_t)p.groups << p.lanes_log, words == 1 ? 4 : words <= 4 ? 2 : 1, &p.bx_log, &grid);
    if (st) return st;
    // (what these kernels write are a layer's constants: what follows starts behind them)
    const auto kernel = words == 1   ? quantize_kernel<T, VEC, 1, 4>
                        : words <= 2 ? quantize_kernel<T, VEC, 2, 2>
                        : words <= 4 ? quantize_kernel<T, VEC, 4, 2>
                                     : quantize_kernel<T, VEC, 0, 1>;
    return dsq_launch(kernel, grid, dim3(256), 0, s, dsq_launch_hooks().pdl, 0, p);
}

template <class T, bool VEC> int dequantize(ValueParams p, cudaStream_t s)
{
    dim3 grid;
    const int st = block_shape(p.N, p.pw, VALUE_ROWS, &p.bx_log, &grid);
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
    p.groups = groups;
    p.group_words = groups == 1 ? p.pw : (int)(group / 8);
    p.lanes_log = p.bx_log = 0;
    cudaStream_t s = (cudaStream_t)stream;
    const bool vec = K % 8 == 0;
    switch (dtype) {
    case DSQ_F32: return vec ? quantize<float, true>(p, s) : quantize<float, false>(p, s);
    case DSQ_BF16: return vec ? quantize<__nv_bfloat16, true>(p, s) : quantize<__nv_bfloat16, false>(p, s);
    default: return vec ? quantize<__half, true>(p, s) : quantize<__half, false>(p, s);
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
    p.bx_log = 0;
    cudaStream_t s = (cudaStream_t)stream;
    const bool vec = K % 8 == 0;
    switch (dtype) {
    case DSQ_F32: return vec ? dequantize<float, true>(p, s) : dequantize<float, false>(p, s);
    case DSQ_BF16: return vec ? dequantize<__nv_bfloat16, true>(p, s) : dequantize<__nv_bfloat16, false>(p, s);
    default: return vec ? dequantize<__half, true>(p, s) : dequantize<__half, false>(p, s);
    }
}

}  // extern "C"
