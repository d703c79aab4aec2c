// Norms of the heads of queries and keys with the position rotation in the same pass, and their
// gradients (what stands between a decoder's q and k products and its attention).
//
//   n = x rstd w,  rstd = 1 / sqrt(mean x^2 + eps)          over the D elements of a head
//   (y1, y2) = (n1 c - n2 s, n2 c + n1 s)                    of the pairs i < R / 2, the rest as it is
// with c, s of the angle position[axis[i]] f[i].  Back: g = the gradient turned by the negative
// angle, grad_x = rstd (g w - n' mean(g w n')) with n' = x rstd, grad_w = sum g n'.
//
// HBM-bound: a head is read once and written once, everything between is in registers.
//   * A unit is 32 bytes of a head (two 16-byte vectors): the first and second elements of the same
//     pairs, so that a turn needs no other lane; L lanes (a power of two) share a head and two sums.
//   * A block takes the heads of some tokens; their cosines and sines are made once a block, in
//     shared memory, one angle for all heads.  An angle is formed and reduced to a quarter turn in
//     binary64 (a position of 2^20 leaves 2^-4 of an angle in binary32).
//   * Blocks of q and blocks of k are apart: a lane keeps the weights (and the sums of their
//     gradient) of its own unit in registers.
//   * Heads or strides that are no multiple of a vector go element by element, 32 lanes a head.
#include "dsq_launch.h"
#include "dsq_ptx.cuh"
#include "dsq_tc_host.h"
#include "dsq_types.cuh"

using namespace dsq_ptx;

namespace {

constexpr int BLOCK = 256, MAX_DIM = 512, MAX_HEADS = 4096, TURN_BYTES = 16384;

struct Tensor {
    const void *x, *gy;           // (gy: backward)
    void *y;                      // forward y, backward grad_x
    const float *w;
    float *part;                  // sums of the weight's gradient, [blocks][D]
    int64_t x_token, x_head, y_token, y_head, g_token, g_head;
    int heads, tile;              // tokens of a tile
    uint32_t heads_inv;           // floor(2^32 / heads) + 1
};

struct Params {
    Tensor t[2];                  // q, k
    const int64_t *pos;
    const float *freq;
    const uint8_t *axis;
    int64_t tokens;
    int q_blocks, k_blocks;
    int D, R, axes, norm, lanes, units;
    float eps, inv_d;
};

// cosine and sine of pos f
__device__ __forceinline__ float2 turn_of(int64_t pos, float f)
{
    const double a = (double)pos * (double)f;
    const double k = rint(a * 0.6366197723675814);           // quarter turns
    // pi / 2 in two parts
    const double r = fma(-k, 6.123233995736766e-17, fma(-k, 1.5707963267948966, a));
    float s, c;
    sincosf((float)r, &s, &c);
    const int q = (int)(fma(-4.0, floor(k * 0.25), k));       // k mod 4
    float2 t;
    t.x = q & 1 ? s : c;
    t.y = q & 1 ? c : s;
    if (q == 1 || q == 2) t.x = -t.x;
    if (q >= 2) t.y = -t.y;
    return t;
}

// Where pair i's turn lies among a token's: units' pairs 2 q, 2 q + 1 side by side over the units, so that the lanes
// of a head read consecutive 16 bytes.
template <int VEC> __device__ __forceinline__ int turn_at(int i, int units)
{
    return VEC == 1 ? i : ((i % VEC) / 2 * units + i / VEC) * 2 + (i & 1);
}

// the turns of `n` tokens from token0 on
template <int VEC> __device__ __forceinline__ void make_turns(const Params &p, int64_t token0, int n, float2 *turns)
{
    const int half = p.R / 2, units = half / VEC;
    for (int e = threadIdx.x; e < n * half; e += BLOCK) {
        const int t = e / half, i = e - t * half;
        const int axis = p.axis ? p.axis[i] : 0;
        float2 v = make_float2(__int_as_float(0x7FC00000), __int_as_float(0x7FC00000));   // (no such axis: NaN)
        if (axis < p.axes) v = turn_of(p.pos[axis * p.tokens + token0 + t], p.freq[i]);
        turns[t * half + turn_at<VEC>(i, units)] = v;
    }
}

template <class T, int VEC> __device__ __forceinline__ void load_vec(const T *p, T (&v)[VEC])
{
    if constexpr (VEC == 1) v[0] = *p;
    else {
        uint4 r;
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
        *reinterpret_cast<uint4 *>(v) = r;
    }
}
template <class T, int VEC> __device__ __forceinline__ void store_vec(T *p, const float *f)
{
    if constexpr (VEC == 1) *p = dsq_from_f32<T>(f[0]);
    else {
        alignas(16) T v[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = dsq_from_f32<T>(f[i]);
        *reinterpret_cast<uint4 *>(p) = *reinterpret_cast<const uint4 *>(v);
    }
}

// where the two vectors of unit u start; which of them exist, whether it is rotated
struct Unit { int a, b; bool has_a, has_b, turned; };
template <int VEC, bool INTER> __device__ __forceinline__ Unit unit_of(const Params &p, int u)
{
    const int turned = p.R / (2 * VEC);
    Unit r;
    r.turned = u < turned;
    if (r.turned) {
        r.a = INTER ? 2 * u * VEC : u * VEC;
        r.b = INTER ? r.a + VEC : r.a + p.R / 2;
    } else {
        r.a = p.R + (u - turned) * 2 * VEC;
        r.b = r.a + VEC;
    }
    r.has_a = r.a < p.D;
    r.has_b = r.b < p.D;
    return r;
}

__device__ __forceinline__ float lanes_sum(float v, int lanes)
{
    for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}
// heads of a tile (tile_of), a bit each
constexpr int MAX_PASSES = 8, MARKS = (MAX_HEADS > BLOCK * MAX_PASSES ? MAX_HEADS : BLOCK * MAX_PASSES) / 32;
// squares, and what is divided by their root, are inside binary32's range
__device__ __forceinline__ bool in_range(float mean) { return mean > 1e-28f && mean < 1e36f; }

// A head whose squares are not (found in the loop, done behind it): by a whole warp in binary64, element by element.  `sums`: the warp's
// sums of the weight's gradient.  Every pair is read and written by one lane.
template <class T, bool BACK> __device__ __noinline__ void wide_head(const Params &p, const Tensor &t, int64_t token, int head,
                                                                     bool inter, float *sums)
{
    const T *x = (const T *)t.x + token * t.x_token + head * t.x_head;
    const T *gy = (const T *)t.gy + token * t.g_token + head * t.g_head;
    T *y = (T *)t.y + token * t.y_token + head * t.y_head;
    const int lane = threadIdx.x & 31, half = p.R / 2;
    // f(element, element | -1, turn) of each pair, then of what is not rotated
    auto each = [&](auto f) {
        for (int i = lane; i < half; i += 32) {
            const int axis = p.axis ? p.axis[i] : 0;
            const float2 turn = axis < p.axes ? turn_of(p.pos[axis * p.tokens + token], p.freq[i])
                                              : make_float2(__int_as_float(0x7FC00000), __int_as_float(0x7FC00000));
            f(inter ? 2 * i : i, inter ? 2 * i + 1 : i + half, turn);
        }
        for (int i = p.R + lane; i < p.D; i += 32) f(i, -1, make_float2(1.f, 0.f));
    };
    auto value = [](const T *from, int i) { return i < 0 ? 0.0 : (double)dsq_to_f32(from[i]); };
    auto weight = [&](int i) { return t.w && i >= 0 ? (double)t.w[i] : 1.0; };
    double sum = 0.0, dot = 0.0;
    each([&](int i, int j, float2 turn) {
        const double a = value(x, i), b = value(x, j);
        sum += a * a + b * b;
        if (BACK) {
            const double ga = value(gy, i), gb = value(gy, j);
            dot += (ga * turn.x + gb * turn.y) * weight(i) * a + (gb * turn.x - ga * turn.y) * weight(j) * b;
        }
    });
    for (int o = 16; o > 0; o >>= 1) {
        sum += __shfl_xor_sync(~0u, sum, o);
        dot += __shfl_xor_sync(~0u, dot, o);
    }
    const double mean = sum / p.D + p.eps;
    const double r = mean > 0.0 || mean != mean ? 1.0 / sqrt(mean) : 0.0, c = dot * r / p.D;
    each([&](int i, int j, float2 turn) {
        const double a = value(x, i) * r, b = value(x, j) * r;
        double o1, o2;
        if (BACK) {
            const double ga = value(gy, i), gb = value(gy, j);
            const double g1 = ga * turn.x + gb * turn.y, g2 = gb * turn.x - ga * turn.y;
            sums[i] += (float)(g1 * a);
            if (j >= 0) sums[j] += (float)(g2 * b);
            o1 = r * (g1 * weight(i) - a * c);
            o2 = r * (g2 * weight(j) - b * c);
        } else {
            const double n1 = a * weight(i), n2 = b * weight(j);
            o1 = n1 * turn.x - n2 * turn.y;
            o2 = n2 * turn.x + n1 * turn.y;
        }
        y[i] = dsq_from_f32<T>((float)o1);
        if (j >= 0) y[j] = dsq_from_f32<T>((float)o2);
    });
}
// the marked heads of a tile, a warp each; marks are cleared
template <class T, bool BACK> __device__ __forceinline__ void wide_heads(const Params &p, const Tensor &t, int64_t token0, int rows,
                                                                         uint32_t *marks, bool inter, float *sums)
{
    const int warp = threadIdx.x >> 5;
    for (int w = warp; 32 * w < rows; w += BLOCK / 32) {
        uint32_t mask = marks[w];
        while (mask) {
            const int row = 32 * w + __ffs(mask) - 1;
            wide_head<T, BACK>(p, t, token0 + row / t.heads, row % t.heads, inter, sums);
            mask &= mask - 1;
        }
        __syncwarp();
        if ((threadIdx.x & 31) == 0) marks[w] = 0u;
    }
}

// A lane's part of a head: U units, element i of vector v of unit u at (2 u + v) VEC + i.
template <class T, int VEC, int U, bool INTER> struct Lane {
    static constexpr int N = 2 * U * VEC;
    Unit unit[U];
    float w[N];
    __device__ __forceinline__ void init(const Params &p, const Tensor &t, int lane)
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            unit[u] = unit_of<VEC, INTER>(p, lane + u * p.lanes);
            if (lane + u * p.lanes >= p.units) unit[u].has_a = unit[u].has_b = unit[u].turned = false;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                w[2 * u * VEC + i] = t.w && unit[u].has_a ? __ldg(t.w + unit[u].a + i) : 1.f;
                w[(2 * u + 1) * VEC + i] = t.w && unit[u].has_b ? __ldg(t.w + unit[u].b + i) : 1.f;
            }
        }
    }
    // (what does not exist is zero)
    __device__ __forceinline__ void load(const T *row, bool on, T (&r)[U][2][VEC]) const
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) r[u][0][i] = r[u][1][i] = dsq_from_f32<T>(0.f);
            if (on && unit[u].has_a) load_vec<T, VEC>(row + unit[u].a, r[u][0]);
            if (on && unit[u].has_b) load_vec<T, VEC>(row + unit[u].b, r[u][1]);
        }
    }
    __device__ __forceinline__ static void values(const T (&r)[U][2][VEC], float (&f)[N])
    {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = dsq_to_f32(r[i / (2 * VEC)][i / VEC % 2][i % VEC]);
    }
    __device__ __forceinline__ void store(T *row, const float (&f)[N]) const
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (unit[u].has_a) store_vec<T, VEC>(row + unit[u].a, f + 2 * u * VEC);
            if (unit[u].has_b) store_vec<T, VEC>(row + unit[u].b, f + (2 * u + 1) * VEC);
        }
    }
    // turns the pairs, forwards (dir = 1) or back (-1)
    __device__ __forceinline__ void turn(float (&f)[N], const float2 *turns, int lane, const Params &p, float dir) const
    {
        const int turned = p.R / (2 * VEC);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!unit[u].turned) continue;
            const int at = lane + u * p.lanes;
#pragma unroll
            for (int j = 0; j < VEC; j += 2) {
                float2 t[2];
                if constexpr (VEC == 1) t[0] = turns[at];
                else {
                    const float4 v = *reinterpret_cast<const float4 *>(turns + (j / 2 * turned + at) * 2);
                    t[0] = make_float2(v.x, v.y);
                    t[1] = make_float2(v.z, v.w);
                }
#pragma unroll
                for (int h = 0; h < (VEC == 1 ? 1 : 2); ++h) {
                    const int i = j + h;                       // the unit's i-th pair
                    float &f1 = f[2 * u * VEC + (INTER ? 2 * i : i)];
                    float &f2 = f[2 * u * VEC + (INTER ? 2 * i + 1 : VEC + i)];
                    const float c = t[h].x, s = t[h].y * dir, a = f1, b = f2;
                    f1 = __fmaf_rn(a, c, -(b * s));
                    f2 = __fmaf_rn(b, c, a * s);
                }
            }
        }
    }
};

// The heads of a tile of tokens, a head to L lanes: which one a thread has, and the next.
struct Place {
    int row, token, head;
    __device__ __forceinline__ void to(const Tensor &t, int r)
    {
        row = r;
        token = t.heads == 1 ? r : (int)__umulhi((uint32_t)r, t.heads_inv);
        head = r - token * t.heads;
    }
};

template <class T, int VEC, int U, bool INTER>
__global__ void __launch_bounds__(BLOCK, U * VEC > 8 ? 2 : 4) heads_fwd_kernel(const __grid_constant__ Params p)
{
    using L = Lane<T, VEC, U, INTER>;
    extern __shared__ __align__(16) float2 turns[];
    __shared__ uint32_t marks[MARKS];
    const bool second = (int)blockIdx.x >= p.q_blocks;
    const Tensor &t = p.t[second];
    const int64_t token0 = (int64_t)(blockIdx.x - (second ? p.q_blocks : 0)) * t.tile;
    const int n = (int)min((int64_t)t.tile, p.tokens - token0), rows = n * t.heads;
    const int lane = threadIdx.x & (p.lanes - 1), step = BLOCK / p.lanes;
    grid_dependency_wait();
    grid_launch_dependents();
    L l;
    l.init(p, t, lane);
    Place at = {};
    T next[U][2][VEC];
    auto load = [&]() {
        l.load((const T *)t.x + (token0 + at.token) * t.x_token + at.head * t.x_head, at.row < rows, next);
    };
    at.to(t, threadIdx.x / p.lanes);
    load();
    bool any = false;
    for (int i = threadIdx.x; i < MARKS; i += BLOCK) marks[i] = 0u;
    make_turns<VEC>(p, token0, n, turns);
    __syncthreads();
    // (a warp's lanes go round together: the sums are over lanes)
    for (int first = (threadIdx.x & ~31) / p.lanes; first < rows; first += step) {
        float f[L::N];
        L::values(next, f);
        const Place here = at;
        bool on = here.row < rows;
        at.to(t, at.row + step);
        load();
        if (p.norm) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < L::N; ++i) sum = __fmaf_rn(f[i], f[i], sum);
            const float mean = __fmaf_rn(lanes_sum(sum, p.lanes), p.inv_d, p.eps);
            const float rstd = 1.f / sqrtf(mean);
            const bool bad = on && !in_range(mean);
            if (bad) {
                if (lane == 0) atomicOr(&marks[here.row >> 5], 1u << (here.row & 31));
                on = false;
                any = true;
            }
#pragma unroll
            for (int i = 0; i < L::N; ++i) f[i] = f[i] * rstd * l.w[i];
        }
        if (on) {
            l.turn(f, turns + here.token * (p.R / 2), lane, p, 1.f);
            l.store((T *)t.y + (token0 + here.token) * t.y_token + here.head * t.y_head, f);
        }
    }
    if (__syncthreads_or(any)) wide_heads<T, false>(p, t, token0, rows, marks, INTER, nullptr);
}

template <class T, int VEC, int U, bool INTER>
__global__ void __launch_bounds__(BLOCK, U * VEC > 8 ? 1 : 2) heads_bwd_kernel(const __grid_constant__ Params p)
{
    using L = Lane<T, VEC, U, INTER>;
    extern __shared__ __align__(16) float2 turns[];
    __shared__ float sums[BLOCK / 32][MAX_DIM];
    __shared__ uint32_t marks[MARKS];
    const bool second = (int)blockIdx.x >= p.q_blocks;
    const Tensor &t = p.t[second];
    const int block = blockIdx.x - (second ? p.q_blocks : 0), blocks = second ? p.k_blocks : p.q_blocks;
    const int lane = threadIdx.x & (p.lanes - 1), step = BLOCK / p.lanes;
    grid_dependency_wait();
    grid_launch_dependents();
    L l;
    l.init(p, t, lane);
    float gw[L::N];
#pragma unroll
    for (int i = 0; i < L::N; ++i) gw[i] = 0.f;
    for (int c = threadIdx.x & 31; c < p.D; c += 32) sums[threadIdx.x >> 5][c] = 0.f;
    for (int i = threadIdx.x; i < MARKS; i += BLOCK) marks[i] = 0u;
    __syncthreads();

    for (int64_t token0 = (int64_t)block * t.tile; token0 < p.tokens; token0 += (int64_t)blocks * t.tile) {
        const int n = (int)min((int64_t)t.tile, p.tokens - token0), rows = n * t.heads;
        Place at = {};
        T next_x[U][2][VEC], next_g[U][2][VEC];
        auto load = [&]() {
            l.load((const T *)t.gy + (token0 + at.token) * t.g_token + at.head * t.g_head, at.row < rows, next_g);
            l.load((const T *)t.x + (token0 + at.token) * t.x_token + at.head * t.x_head, p.norm && at.row < rows, next_x);
        };
        at.to(t, threadIdx.x / p.lanes);
        load();
        bool any = false;
        make_turns<VEC>(p, token0, n, turns);
        __syncthreads();
        for (int first = (threadIdx.x & ~31) / p.lanes; first < rows; first += step) {
            float g[L::N], x[L::N];
            L::values(next_g, g);
            L::values(next_x, x);
            const Place here = at;
            bool on = here.row < rows;
            at.to(t, at.row + step);
            load();
            if (on) l.turn(g, turns + here.token * (p.R / 2), lane, p, -1.f);
            if (p.norm) {
                float sum = 0.f, dot = 0.f;
#pragma unroll
                for (int i = 0; i < L::N; ++i) {
                    sum = __fmaf_rn(x[i], x[i], sum);
                    dot = __fmaf_rn(g[i] * l.w[i], x[i], dot);
                }
                sum = lanes_sum(sum, p.lanes);
                dot = lanes_sum(dot, p.lanes);
                const float mean = __fmaf_rn(sum, p.inv_d, p.eps), rstd = 1.f / sqrtf(mean);
                const bool bad = on && !in_range(mean);
                if (bad) {
                    if (lane == 0) atomicOr(&marks[here.row >> 5], 1u << (here.row & 31));
                    on = false;
                    any = true;
                }
                if (on) {
                    const float c = dot * rstd * p.inv_d;
#pragma unroll
                    for (int i = 0; i < L::N; ++i) {
                        const float m = x[i] * rstd;
                        gw[i] = __fmaf_rn(g[i], m, gw[i]);
                        g[i] = rstd * __fmaf_rn(-m, c, g[i] * l.w[i]);
                    }
                }
            }
            if (on) l.store((T *)t.y + (token0 + here.token) * t.y_token + here.head * t.y_head, g);
        }
        // (and the turns have been read)
        if (__syncthreads_or(any)) wide_heads<T, true>(p, t, token0, rows, marks, INTER, sums[threadIdx.x >> 5]);
    }
    if (!t.part) return;
    // the block's sums: over the heads of a warp, then the warps, in one order
    __syncwarp();
#pragma unroll
    for (int i = 0; i < L::N; ++i) {
        float s = gw[i];
        for (int o = 16; o >= p.lanes; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
        const Unit &u = l.unit[i / (2 * VEC)];
        const bool b = i / VEC % 2;
        if ((threadIdx.x & 31) < p.lanes && (b ? u.has_b : u.has_a)) sums[threadIdx.x >> 5][(b ? u.b : u.a) + i % VEC] += s;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < p.D; c += BLOCK) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < BLOCK / 32; ++w) s += sums[w][c];
        t.part[(int64_t)block * p.D + c] = s;
    }
}

// grad_w[c] = sum over the blocks of their sums, in one order: a warp a column, of q (blockIdx.y = 0) or k
struct SumParams {
    const float *part[2];
    float *out[2];
    int blocks[2], D;
};
__global__ void __launch_bounds__(1024) heads_sum_kernel(const SumParams p)
{
    __shared__ float s[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, col = blockIdx.x * 32 + x;
    const float *part = p.part[blockIdx.y];
    const int rows = p.blocks[blockIdx.y];
    grid_dependency_wait();
    grid_launch_dependents();
    if (!p.out[blockIdx.y]) return;
    float a = 0.f;
    if (col < p.D)
        for (int r = y; r < rows; r += 256) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = r + 32 * i < rows ? __ldcg(part + (int64_t)(r + 32 * i) * p.D + col) : 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) a += v[i];
        }
    s[y][x] = a;
    __syncthreads();
    a = s[x][y];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a += __shfl_xor_sync(~0u, a, o);
    if (x == 0 && blockIdx.x * 32 + y < p.D) p.out[blockIdx.y][blockIdx.x * 32 + y] = a;
}

// ---- host ----------------------------------------------------------------------------
// A head goes in vectors where its pairs and all its rows do.
bool in_vectors(const void *p, int64_t token, int64_t head, int vec, int size)
{
    return dsq_aligned16(p) && token % vec == 0 && head % vec == 0 && vec * size == 16;
}

bool aligned_to(const void *p, int size) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(size - 1)) == 0; }

// rows that are written lie apart
bool apart(int64_t tokens, int64_t heads, int64_t token, int64_t head, int64_t D)
{
    if (token < 0 || head < 0) return false;
    if (tokens == 1) return heads == 1 || head >= D;
    if (heads == 1) return token >= D;
    return (head >= D && (token - D) / head >= heads - 1 && token >= D) ||
           (token >= D && (head - D) / token >= tokens - 1 && head >= D);
}

int check_rotary(const dsq_rotary_t *r, int64_t tokens, int dtype, float eps)
{
    if (!r || !r->positions || (r->rot_dim > 0 && !r->inv_freq)) return DSQ_ERR_NULL;
    if (!dsq_is_float_type(dtype)) return DSQ_ERR_UNSUPPORTED;
    if (tokens <= 0 || r->head_dim <= 0 || r->rot_dim < 0 || r->rot_dim > r->head_dim || r->rot_dim % 2 ||
        r->axes < 1)
        return DSQ_ERR_SHAPE;
    if (r->head_dim > MAX_DIM || r->axes > 255 || tokens > (int64_t)1 << 31) return DSQ_ERR_SIZE;
    if (r->head_dim % 2) return DSQ_ERR_UNSUPPORTED;
    if (!dsq_finite(eps) || eps < 0.f) return DSQ_ERR_RANGE;
    if (!aligned_to(r->positions, 8) || !aligned_to(r->inv_freq, 4)) return DSQ_ERR_ALIGN;
    return DSQ_OK;
}

template <class T> constexpr int vec_of() { return 16 / (int)sizeof(T); }

// Fills in what depends on the vectors' length.
void set_lanes(Params &p, int vec)
{
    const int turned = p.R / (2 * vec), rest = (p.D - p.R + 2 * vec - 1) / (2 * vec);
    p.units = turned + rest;
    p.lanes = 1;
    while (p.lanes < p.units && p.lanes < 32) p.lanes *= 2;
}

// Tokens of a tile: `passes` rounds of a block's lanes, as far as their turns have room.
int tile_of(const Params &p, int64_t heads, int passes)
{
    const int rows = BLOCK / p.lanes * passes;
    int64_t tile = rows / heads;
    const int64_t room = p.R > 0 ? TURN_BYTES / (p.R * 4) : tile;
    if (tile > room) tile = room;
    if (tile > p.tokens) tile = p.tokens;
    return tile < 1 ? 1 : (int)tile;
}

size_t turn_bytes(const Params &p)
{
    const int tile = p.t[0].tile > p.t[1].tile ? p.t[0].tile : p.t[1].tile;
    return (size_t)tile * p.R * 4 + 16;
}

constexpr int SUM_BLOCKS_PER_SM = 4;

template <class T, int VEC, int U, bool INTER> int launch(Params &p, bool back, cudaStream_t s)
{
    const int pdl = dsq_launch_hooks().pdl;
    const int64_t sms = dsq_sm_count() > 0 ? dsq_sm_count() : 148;
    const int64_t rows = p.tokens * (p.t[0].heads + p.t[1].heads), round = BLOCK / p.lanes;
    if (!back) {
        // as many rounds a block as leave some blocks for every place on an SM
        int passes = (int)(rows / (round * sms * 16));
        passes = passes < 1 ? 1 : passes > MAX_PASSES ? MAX_PASSES : passes;
        int64_t blocks[2] = {0, 0};
        for (int i = 0; i < 2; ++i) {
            if (!p.t[i].heads) continue;
            p.t[i].tile = tile_of(p, p.t[i].heads, passes);
            blocks[i] = (p.tokens + p.t[i].tile - 1) / p.t[i].tile;
        }
        if (blocks[0] + blocks[1] > 0x7FFFFFFF) return DSQ_ERR_SIZE;
        p.q_blocks = (int)blocks[0];
        p.k_blocks = (int)blocks[1];
        return dsq_launch(heads_fwd_kernel<T, VEC, U, INTER>, dim3((unsigned)(blocks[0] + blocks[1])), dim3(BLOCK),
                          turn_bytes(p), s, pdl, 0, p);
    }
    // what is resident together, shared among q and k as their rows are
    int64_t most = sms * SUM_BLOCKS_PER_SM, blocks[2] = {0, 0};
    for (int i = 0; i < 2; ++i) {
        if (!p.t[i].heads) continue;
        p.t[i].tile = tile_of(p, p.t[i].heads, 2);
        const int64_t tiles = (p.tokens + p.t[i].tile - 1) / p.t[i].tile;
        int64_t share = most * p.t[i].heads / (p.t[0].heads + p.t[1].heads);
        if (share < 1) share = 1;
        blocks[i] = tiles < share ? tiles : share;
    }
    p.q_blocks = (int)blocks[0];
    p.k_blocks = (int)blocks[1];
    if (p.t[1].part) p.t[1].part = p.t[0].part + blocks[0] * p.D;
    return dsq_launch(heads_bwd_kernel<T, VEC, U, INTER>, dim3((unsigned)(blocks[0] + blocks[1])), dim3(BLOCK),
                      turn_bytes(p), s, pdl, 0, p);
}

template <class T> int pick(Params &p, bool back, bool vectors, bool inter, cudaStream_t s)
{
    constexpr int V = vec_of<T>();
    set_lanes(p, vectors ? V : 1);
    const int per_lane = (p.units + p.lanes - 1) / p.lanes;
#define FORM(VEC, U) return inter ? launch<T, VEC, U, true>(p, back, s) : launch<T, VEC, U, false>(p, back, s)
    if (vectors) {
        if constexpr (V == 4) {
            if (per_lane == 2) FORM(V, 2);
        }
        FORM(V, 1);
    }
    if (per_lane <= 2) FORM(1, 2);
    FORM(1, 8);
#undef FORM
}

int start(Params &p, bool back, bool vectors, bool inter, int dtype, cudaStream_t s)
{
    switch (dtype) {
    case DSQ_F32: return pick<float>(p, back, vectors, inter, s);
    case DSQ_BF16: return pick<__nv_bfloat16>(p, back, vectors, inter, s);
    default: return pick<__half>(p, back, vectors, inter, s);
    }
}

void fill(Params &p, const dsq_rotary_t *r, int64_t tokens, int norm, float eps)
{
    p = Params{};
    p.pos = r->positions; p.freq = r->inv_freq; p.axis = r->axis;
    p.tokens = tokens;
    p.D = r->head_dim; p.R = r->rot_dim; p.axes = r->axes;
    p.norm = norm != 0;
    p.eps = eps; p.inv_d = (float)(1.0 / r->head_dim);
}

// whether pairs and the rest are whole vectors
bool whole(const Params &p, int vec) { return p.R / 2 % vec == 0 && (p.D - p.R) % vec == 0; }

int check_heads(int64_t heads, int64_t tokens)
{
    if (heads <= 0) return DSQ_ERR_SHAPE;
    return heads > MAX_HEADS || tokens * heads > (int64_t)1 << 40 ? DSQ_ERR_SIZE : DSQ_OK;
}

}  // namespace

extern "C" {

int dsq_headnorm_fwd(const dsq_heads_t *q, const dsq_heads_t *k, int64_t tokens, const dsq_rotary_t *rotary,
                     int norm, float eps, int dtype, void *stream)
{
    if (!q || !q->x || !q->y || (k && (!k->x || !k->y))) return DSQ_ERR_NULL;
    int st = check_rotary(rotary, tokens, dtype, eps);
    if (st) return st;
    Params p;
    fill(p, rotary, tokens, norm, eps);
    const int size = dtype == DSQ_F32 ? 4 : 2, vec = 16 / size;
    bool vectors = whole(p, vec);
    const dsq_heads_t *in[2] = {q, k};
    for (int i = 0; i < 2; ++i) {
        const dsq_heads_t *h = in[i];
        if (!h) continue;
        st = check_heads(h->heads, tokens);
        if (st) return st;
        if (h->weight && !norm) return DSQ_ERR_UNSUPPORTED;
        if (!aligned_to(h->x, size) || !aligned_to(h->y, size) || !aligned_to(h->weight, 4)) return DSQ_ERR_ALIGN;
        if (!apart(tokens, h->heads, h->y_token, h->y_head, p.D)) return DSQ_ERR_SHAPE;
        Tensor &t = p.t[i];
        t.x = h->x; t.y = h->y; t.w = h->weight;
        t.x_token = h->x_token; t.x_head = h->x_head; t.y_token = h->y_token; t.y_head = h->y_head;
        t.heads = (int)h->heads;
        t.heads_inv = h->heads > 1 ? (uint32_t)((1ull << 32) / (uint64_t)h->heads + 1) : 0u;
        vectors = vectors && in_vectors(h->x, h->x_token, h->x_head, vec, size) &&
                  in_vectors(h->y, h->y_token, h->y_head, vec, size);
    }
    return start(p, false, vectors, rotary->interleaved != 0, dtype, (cudaStream_t)stream);
}

size_t dsq_headnorm_bwd_workspace_bytes(int64_t head_dim)
{
    if (head_dim <= 0 || head_dim > MAX_DIM) return DSQ_WS_BYTES;
    const int sms = dsq_sm_count() > 0 ? dsq_sm_count() : 148;
    return DSQ_WS_BYTES + (size_t)(sms * SUM_BLOCKS_PER_SM + 2) * (size_t)head_dim * 4;
}

int dsq_headnorm_bwd(const dsq_heads_grad_t *q, const dsq_heads_grad_t *k, int64_t tokens,
                     const dsq_rotary_t *rotary, int norm, float eps, int dtype, void *workspace,
                     size_t ws_bytes, void *stream)
{
    const dsq_heads_grad_t *in[2] = {q, k};
    if (!q) return DSQ_ERR_NULL;
    bool sums = false;
    for (const dsq_heads_grad_t *h : in) {
        if (!h) continue;
        if (!h->grad_y || !h->grad_x || (norm && !h->x)) return DSQ_ERR_NULL;
        sums = sums || h->grad_weight;
    }
    if (sums && !workspace) return DSQ_ERR_NULL;
    int st = check_rotary(rotary, tokens, dtype, eps);
    if (st) return st;
    Params p;
    fill(p, rotary, tokens, norm, eps);
    const int size = dtype == DSQ_F32 ? 4 : 2, vec = 16 / size;
    bool vectors = whole(p, vec);
    SumParams sp = {};
    for (int i = 0; i < 2; ++i) {
        const dsq_heads_grad_t *h = in[i];
        if (!h) continue;
        st = check_heads(h->heads, tokens);
        if (st) return st;
        if ((h->weight || h->grad_weight) && !norm) return DSQ_ERR_UNSUPPORTED;
        if (!aligned_to(h->grad_y, size) || !aligned_to(h->x, size) || !aligned_to(h->grad_x, size) ||
            !aligned_to(h->weight, 4) || !aligned_to(h->grad_weight, 4))
            return DSQ_ERR_ALIGN;
        if (!apart(tokens, h->heads, h->gx_token, h->gx_head, p.D)) return DSQ_ERR_SHAPE;
        Tensor &t = p.t[i];
        t.gy = h->grad_y; t.x = h->x; t.y = h->grad_x; t.w = h->weight;
        t.g_token = h->gy_token; t.g_head = h->gy_head;
        t.x_token = h->x_token; t.x_head = h->x_head; t.y_token = h->gx_token; t.y_head = h->gx_head;
        t.heads = (int)h->heads;
        t.heads_inv = h->heads > 1 ? (uint32_t)((1ull << 32) / (uint64_t)h->heads + 1) : 0u;
        // (sums of both are made where either is wanted)
        t.part = sums ? (float *)((char *)workspace + DSQ_WS_BYTES) : nullptr;
        sp.out[i] = h->grad_weight;
        vectors = vectors && in_vectors(h->grad_y, h->gy_token, h->gy_head, vec, size) &&
                  in_vectors(h->grad_x, h->gx_token, h->gx_head, vec, size) &&
                  (!norm || in_vectors(h->x, h->x_token, h->x_head, vec, size));
    }
    if (sums && !dsq_aligned16(workspace)) return DSQ_ERR_ALIGN;
    if (sums && ws_bytes < dsq_headnorm_bwd_workspace_bytes(p.D)) return DSQ_ERR_SIZE;
    st = start(p, true, vectors, rotary->interleaved != 0, dtype, (cudaStream_t)stream);
    if (st || !sums) return st;
    for (int i = 0; i < 2; ++i) sp.part[i] = p.t[i].part;
    sp.blocks[0] = p.q_blocks; sp.blocks[1] = p.k_blocks;
    sp.D = p.D;
    return dsq_launch(heads_sum_kernel, dim3((unsigned)((p.D + 31) / 32), 2), dim3(1024), 0, (cudaStream_t)stream,
                      dsq_launch_hooks().pdl, 0, sp);
}

}  // extern "C"
