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
//     pairs, so that a turn needs no other lane; L lanes (a power of two), a team, share a head and two sums.
//   * A team takes a token's heads one after the other (all of them, or a part where there are few
//     tokens): a lane has the same pairs of all of them, makes their cosines and sines itself and
//     keeps them in registers; nothing goes through shared memory and no team waits for another.
//     (With a table a block in shared memory, for all heads: 16384 tokens of 32 + 8 heads of 128 in bf16 67 us.)
//     An angle is formed and reduced to a quarter turn in binary64 (a position of 2^20 leaves 2^-4 of
//     an angle in binary32).
//   * Backwards teams take either heads of q or of k, and a lane keeps the sums of the weights' gradient of its
//     pairs in registers; blocks leave theirs in the workspace, a second kernel adds them in one order.
//   * Heads or strides that are no multiple of a vector go element by element, 32 lanes a head.
// 16384 tokens of 32 + 8 heads of 128 in bf16: 60 us, 5.6 TB/s; what is missing are pages of memory left and entered again (a
// warp that has a token's heads in a row, 60; a team a token, 67).  Backwards 8192 tokens of 16 + 16 heads of 64: 22 us, 4.5 TB/s:
// three blocks an SM (168 registers), whose chains of loads, sums over lanes and a root take turns; with a ring of copies in
// shared memory, three heads ahead, 27, with four blocks and spilled registers 32.
#include "dsq_launch.h"
#include "dsq_pairs.cuh"
#include "dsq_ptx.cuh"
#include "dsq_tc_host.h"
#include "dsq_types.cuh"

using namespace dsq_ptx;

namespace {

constexpr int BLOCK = 128, MAX_DIM = 512, MAX_HEADS = 4096;

struct Tensor {
    const void *x, *gy;           // (gy: backward)
    void *y;                      // forward y, backward grad_x
    const float *w;
    float *part;                  // sums of the weight's gradient, [blocks][D]
    int64_t x_token, x_head, y_token, y_head, g_token, g_head;
    int heads;
    int parts, per_part;          // of a token's heads (forward: of q's and k's together, in t[0])
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

// Cosine and sine of pos f: the angle and what it is beyond a whole number of quarter turns in binary64 (below 2^50, else
// NaN: binary64 has no fourth of a turn left then), then the two series at most pi / 4 away from 0, whose first terms left out are
// below 2^-29.
__device__ __forceinline__ float2 turn_of(int64_t pos, float f)
{
    constexpr double WHOLE = 6755399441055744.0;              // 1.5 2^52: the sum's low bits are the whole number
    const double a = (double)pos * (double)f, k1 = fma(a, 0.6366197723675814, WHOLE), k = k1 - WHOLE;
    // pi / 2 in two parts
    float r = (float)fma(-k, 6.123233995736766e-17, fma(-k, 1.5707963267948966, a));
    if (!(fabs(a) < 1125899906842624.0)) r = __int_as_float(0x7FC00000);
    const int q = __double2loint(k1) & 3;
    const float x = r * r;
    float c = __fmaf_rn(x, -1.f / 3628800.f, 1.f / 40320.f);
    c = __fmaf_rn(x, c, -1.f / 720.f);
    c = __fmaf_rn(x, c, 1.f / 24.f);
    c = __fmaf_rn(x, c, -0.5f);
    c = __fmaf_rn(x, c, 1.f);
    float s = __fmaf_rn(x, 1.f / 362880.f, -1.f / 5040.f);
    s = __fmaf_rn(x, s, 1.f / 120.f);
    s = __fmaf_rn(x, s, -1.f / 6.f);
    s = __fmaf_rn(x * r, s, r);
    float2 t;
    t.x = q & 1 ? s : c;
    t.y = q & 1 ? c : s;
    if (q == 1 || q == 2) t.x = -t.x;
    if (q >= 2) t.y = -t.y;
    return t;
}

// a vector as it lies in memory, its elements two by two, and back
template <class T, int VEC> struct Raw { uint4 v; };
template <class T> struct Raw<T, 1> { T v; };
template <class T, int VEC> __device__ __forceinline__ void load_vec(const T *p, Raw<T, VEC> &r)
{
    if constexpr (VEC == 1) r.v = *p;
    else
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(r.v.x), "=r"(r.v.y), "=r"(r.v.z), "=r"(r.v.w) : "l"(p));
}
template <class T, int VEC> __device__ __forceinline__ void clear(Raw<T, VEC> &r)
{
    if constexpr (VEC == 1) r.v = dsq_from_f32<T>(0.f);
    else r.v = make_uint4(0u, 0u, 0u, 0u);
}
template <class T, int VEC> __device__ __forceinline__ void unpack(const Raw<T, VEC> &r, float *f)
{
    if constexpr (VEC == 1) f[0] = dsq_to_f32(r.v);
    else if constexpr (sizeof(T) == 4) {
        f[0] = __uint_as_float(r.v.x); f[1] = __uint_as_float(r.v.y);
        f[2] = __uint_as_float(r.v.z); f[3] = __uint_as_float(r.v.w);
    } else {
        DsqRaw8<T> raw;
        raw.v[0] = r.v;
        float v[8];
        dsq_unpack8(raw, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = v[i];
    }
}
template <class T, int VEC> __device__ __forceinline__ void store_vec(T *p, const float *f)
{
    if constexpr (VEC == 1) *p = dsq_from_f32<T>(f[0]);
    else if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
    else
        *reinterpret_cast<uint4 *>(p) = make_uint4(dsq_pair(f[0], f[1], T()), dsq_pair(f[2], f[3], T()),
                                                   dsq_pair(f[4], f[5], T()), dsq_pair(f[6], f[7], T()));
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

template <int L> __device__ __forceinline__ int lanes_of(const Params &p) { return L ? L : p.lanes; }
template <int L> __device__ __forceinline__ float lanes_sum(float v, int lanes)
{
    if (L) {
#pragma unroll
        for (int o = L >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    } else {
        for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    }
    return v;
}
// squares, and what is divided by their root, are inside binary32's range
__device__ __forceinline__ bool in_range(float mean) { return mean > 1e-28f && mean < 1e36f; }
// Backwards, too, the products of the gradient and x: c is their mean over the root.  (Finite sums leave every product finite; what
// products lose below 2^-149 is, times rstd below 10^4, below the rounding of gradients from 2^-108 on.)
__device__ __forceinline__ bool in_range(float mean, float c) { return mean > 1e-8f && mean < 1e36f && fabsf(c) < 1e36f; }

// A head whose squares are not: by a whole warp in binary64, element by element.  `sums`: the warp's
// sums of the weight's gradient.  Every pair is read and written by one lane.
template <class T, bool BACK> __device__ __forceinline__ void wide_head(const Params &p, const Tensor &t, int64_t token, int head,
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
// Heads that are done behind the loop, a bit each, a row of words a team.  A row's heads are those of a team's part.
constexpr int MARKS = 2048;
__device__ __forceinline__ uint32_t *marks_of(uint32_t *marks, int lanes, int per_part)
{
    return marks + threadIdx.x / lanes * ((per_part + 31) >> 5);
}
// the marked heads of a warp's teams, whose parts begin at (token, first); clears the marks
template <class T, bool BACK> __device__ __noinline__ void wide_heads(const Params &p, const Tensor &t, uint32_t *marks, int lanes,
                                                                      int per_part, int64_t token, int first, bool inter, float *sums)
{
    const int words = (per_part + 31) >> 5;
    __syncwarp();
    for (int from = 0; from < 32; from += lanes) {
        const int64_t tk = __shfl_sync(~0u, token, from);
        const int h0 = __shfl_sync(~0u, first, from);
        uint32_t *row = marks + ((threadIdx.x & ~31) + from) / lanes * words;
        for (int w = 0; w < words; ++w) {
            uint32_t mask = row[w];
            while (mask) {
                const int h = h0 + 32 * w + __ffs(mask) - 1;
                // (forward: of q, then of k)
                const bool second = !BACK && h >= p.t[0].heads;
                wide_head<T, BACK>(p, BACK ? t : p.t[second], tk, second ? h - p.t[0].heads : h, inter, sums);
                mask &= mask - 1;
            }
            __syncwarp();
            if ((threadIdx.x & 31) == 0) row[w] = 0u;
        }
    }
    __syncwarp();
}

// L: lanes of a head, each with all its units and all of them turned; 0: p.lanes, any.
template <class T, int VEC, int U, bool INTER, int L> struct Lane {
    static constexpr int N = 2 * U * VEC, P = N / 2;
    Unit unit[U];
    DsqPair w[P];
    // cosines and sines of the pairs (not turned: 1 and 0), two by two where a unit has more than one
    float c[P], s[P];
    __device__ __forceinline__ void init(const Params &p, int lane)
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            unit[u] = unit_of<VEC, INTER>(p, lane + u * lanes_of<L>(p));
            if (L) unit[u].has_a = unit[u].has_b = unit[u].turned = true;
            else if (lane + u * p.lanes >= p.units) unit[u].has_a = unit[u].has_b = unit[u].turned = false;
        }
    }
    __device__ __forceinline__ void weights(const float *from)
    {
        float v[N];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                v[2 * u * VEC + i] = from && unit[u].has_a ? __ldg(from + unit[u].a + i) : 1.f;
                v[(2 * u + 1) * VEC + i] = from && unit[u].has_b ? __ldg(from + unit[u].b + i) : 1.f;
            }
#pragma unroll
        for (int i = 0; i < P; ++i) w[i] = dsq_pair_of(v[2 * i], v[2 * i + 1]);
    }
    __device__ __forceinline__ float2 turn_at(const Params &p, int64_t token, int lane, int u, int i) const
    {
        if (!unit[u].turned) return make_float2(1.f, 0.f);
        const int pair = (lane + u * lanes_of<L>(p)) * VEC + i, axis = p.axis ? __ldg(p.axis + pair) : 0;
        if (axis < p.axes) return turn_of(__ldg(p.pos + axis * p.tokens + token), __ldg(p.freq + pair));
        return make_float2(__int_as_float(0x7FC00000), __int_as_float(0x7FC00000));       // (no such axis)
    }
    // SHARED: all teams of the warp have the token, and each makes its share of the turns
    template <bool SHARED> __device__ __forceinline__ void turns(const Params &p, int64_t token, int lane)
    {
        constexpr int TEAMS = L ? 32 / L : 2, BY = SHARED ? (TEAMS < VEC ? TEAMS : VEC) : 1;   // (any: two teams at least)
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < VEC; i += BY) {
                if constexpr (BY == 1) {
                    const float2 t = turn_at(p, token, lane, u, i);
                    c[u * VEC + i] = t.x;
                    s[u * VEC + i] = t.y;
                } else {
                    const int lanes = lanes_of<L>(p), team = (threadIdx.x & 31) / lanes;
                    const float2 t = turn_at(p, token, lane, u, i + team % BY);
#pragma unroll
                    for (int k = 0; k < BY; ++k) {
                        c[u * VEC + i + k] = __shfl_sync(~0u, t.x, k * lanes + lane);
                        s[u * VEC + i + k] = __shfl_sync(~0u, t.y, k * lanes + lane);
                    }
                }
            }
    }
    // (what does not exist is zero)
    __device__ __forceinline__ void load(const T *row, bool on, Raw<T, VEC> (&r)[U][2]) const
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (L) {                                           // (rows behind the last: whatever is there is not used)
                if (on) {
                    load_vec(row + unit[u].a, r[u][0]);
                    load_vec(row + unit[u].b, r[u][1]);
                }
                continue;
            }
            clear(r[u][0]);
            clear(r[u][1]);
            if (on && unit[u].has_a) load_vec(row + unit[u].a, r[u][0]);
            if (on && unit[u].has_b) load_vec(row + unit[u].b, r[u][1]);
        }
    }
    __device__ __forceinline__ static void values(const Raw<T, VEC> (&r)[U][2], DsqPair (&f)[P])
    {
        float v[N];
#pragma unroll
        for (int i = 0; i < 2 * U; ++i) unpack(r[i / 2][i % 2], v + i * VEC);
#pragma unroll
        for (int i = 0; i < P; ++i) f[i] = dsq_pair_of(v[2 * i], v[2 * i + 1]);
    }
    __device__ __forceinline__ void store(T *row, const DsqPair (&f)[P]) const
    {
        float v[N];
#pragma unroll
        for (int i = 0; i < P; ++i) dsq_halves(f[i], v[2 * i], v[2 * i + 1]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (L || unit[u].has_a) store_vec<T, VEC>(row + unit[u].a, v + 2 * u * VEC);
            if (L || unit[u].has_b) store_vec<T, VEC>(row + unit[u].b, v + (2 * u + 1) * VEC);
        }
    }
    // turns the pairs, forwards or back
    template <bool BACK> __device__ __forceinline__ void turn(DsqPair (&f)[P]) const
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!L && !unit[u].turned) continue;
            if constexpr (VEC == 1 || INTER) {                 // f[i] is a pair
#pragma unroll
                for (int i = u * VEC; i < (u + 1) * VEC; ++i) {
                    float a, b;
                    dsq_halves(f[i], a, b);
                    const float sn = BACK ? -s[i] : s[i];
                    f[i] = dsq_pair_of(__fmaf_rn(a, c[i], -(b * sn)), __fmaf_rn(b, c[i], a * sn));
                }
            } else {                                           // first and second elements VEC / 2 of these apart
#pragma unroll
                for (int i = 0; i < VEC; i += 2) {
                    float a0, a1, b0, b1;
                    DsqPair &x = f[u * VEC + i / 2], &y = f[u * VEC + VEC / 2 + i / 2];
                    dsq_halves(x, a0, a1);
                    dsq_halves(y, b0, b1);
                    const int k = u * VEC + i;
                    const float s0 = BACK ? -s[k] : s[k], s1 = BACK ? -s[k + 1] : s[k + 1];
                    x = dsq_pair_of(__fmaf_rn(a0, c[k], -(b0 * s0)), __fmaf_rn(a1, c[k + 1], -(b1 * s1)));
                    y = dsq_pair_of(__fmaf_rn(b0, c[k], a0 * s0), __fmaf_rn(b1, c[k + 1], a1 * s1));
                }
            }
        }
    }
};

__device__ __forceinline__ float sum_of(DsqPair v)
{
    float a, b;
    dsq_halves(v, a, b);
    return a + b;
}

// rows on their way ahead of the one at hand; resident blocks of the backward kernel
constexpr int AHEAD = 2, BACK_BLOCKS = 3;

// WARP: the teams of a warp take a token's heads in turn (they lie side by side in memory), else each team has
// a token's of its own.
template <class T, int VEC, int U, bool INTER, int L_, bool WARP>
__global__ void __launch_bounds__(BLOCK, 2 * U * VEC > 16 ? 3 : 5) heads_fwd_kernel(const __grid_constant__ Params p)
{
    using L = Lane<T, VEC, U, INTER, L_>;
    __shared__ uint32_t marks[MARKS];
    const int lanes = lanes_of<L_>(p), lane = threadIdx.x & (lanes - 1), by = WARP ? 32 / lanes : 1;
    const int64_t thread = (int64_t)blockIdx.x * BLOCK + threadIdx.x, item = WARP ? thread >> 5 : thread / lanes;
    const int parts = p.t[0].parts, per_part = p.t[0].per_part, q_heads = p.t[0].heads, heads = q_heads + p.t[1].heads;
    const int64_t token = parts == 1 ? item : item / parts;
    const int begin = parts == 1 ? 0 : (int)(item - token * parts) * per_part;
    const int last = token < p.tokens ? min(begin + per_part, heads) : begin, first = begin + (WARP ? (threadIdx.x & 31) / lanes : 0);
    uint32_t *bad_heads = marks_of(marks, lanes, per_part);
    bool any = false;
    for (int w = lane; 32 * w < per_part; w += lanes) bad_heads[w] = 0u;
    __syncwarp();
    grid_dependency_wait();
    grid_launch_dependents();
    L l;
    l.init(p, lane);
    Raw<T, VEC> next[AHEAD][U][2];
    // the head whose load is next and the one at hand, those of k behind those of q
    int ahead = first, head = first;
    const T *x;
    T *y;
    auto x_of = [&]() {
        const Tensor &t = p.t[ahead >= q_heads];
        x = (const T *)t.x + token * t.x_token + (ahead >= q_heads ? ahead - q_heads : ahead) * t.x_head;
    };
    auto y_of = [&]() {
        const Tensor &t = p.t[head >= q_heads];
        y = (T *)t.y + token * t.y_token + (head >= q_heads ? head - q_heads : head) * t.y_head;
        l.weights(t.w);
    };
    if (first < last) {
        x_of();
        y_of();
    }
    auto load = [&](Raw<T, VEC> (&r)[U][2]) {
        l.load(x, ahead < last, r);
        const bool of_q = ahead < q_heads;
        ahead += by;
        if (of_q && ahead >= q_heads) {
            if (ahead < last) x_of();
        } else {
            x += by * p.t[!of_q].x_head;
        }
    };
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) load(next[a]);
    if (WARP || first < last) l.template turns<WARP>(p, token < p.tokens ? token : 0, lane);
    // (a warp's teams go round together: the sums are over lanes)
    for (int i = 0; i < per_part; i += AHEAD * by) {
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            if (i + a * by >= per_part) break;
            DsqPair f[L::P];
            L::values(next[a], f);
            load(next[a]);
            bool on = head < last;
            if (p.norm) {
                DsqPair sum = 0ull;
#pragma unroll
                for (int k = 0; k < L::P; ++k) sum = dsq_pair_fma(f[k], f[k], sum);
                const float mean = __fmaf_rn(lanes_sum<L_>(sum_of(sum), lanes), p.inv_d, p.eps);
                const float rstd = rsqrtf(mean);
                const bool bad = on && !in_range(mean);
                if (bad) {
                    if (lane == 0) bad_heads[(head - begin) >> 5] |= 1u << ((head - begin) & 31);
                    any = true;
                    on = false;
                }
                const DsqPair r = dsq_pair_of(rstd, rstd);
#pragma unroll
                for (int k = 0; k < L::P; ++k) f[k] = dsq_pair_mul(dsq_pair_mul(f[k], r), l.w[k]);
            }
            if (on) {
                l.template turn<false>(f);
                l.store(y, f);
            }
            const bool of_q = head < q_heads;
            head += by;
            if (of_q && head >= q_heads) {
                if (head < last) y_of();
            } else {
                y += by * p.t[!of_q].y_head;
            }
        }
    }
    if (__any_sync(~0u, any)) wide_heads<T, false>(p, p.t[0], marks, lanes, per_part, token, begin, INTER, nullptr);
}

template <class T, int VEC, int U, bool INTER, int L_, bool WARP>
__global__ void __launch_bounds__(BLOCK, 2 * U * VEC > 16 ? 2 : BACK_BLOCKS) heads_bwd_kernel(const __grid_constant__ Params p)
{
    using L = Lane<T, VEC, U, INTER, L_>;
    __shared__ float sums[BLOCK / 32][MAX_DIM];
    __shared__ uint32_t marks[MARKS];
    const bool second = (int)blockIdx.x >= p.q_blocks;
    const Tensor &t = p.t[second];
    const int block = blockIdx.x - (second ? p.q_blocks : 0), blocks = second ? p.k_blocks : p.q_blocks;
    const int lanes = lanes_of<L_>(p), lane = threadIdx.x & (lanes - 1), by = WARP ? 32 / lanes : 1;
    const int of_warp = WARP ? (threadIdx.x & 31) / lanes : 0, per_item = WARP ? 32 : lanes;
    const int64_t items = p.tokens * t.parts, step = (int64_t)blocks * BLOCK / per_item;
    float *mine = sums[threadIdx.x >> 5];
    for (int c = threadIdx.x & 31; c < p.D; c += 32) mine[c] = 0.f;
    uint32_t *bad_heads = marks_of(marks, lanes, t.per_part);
    for (int w = lane; 32 * w < t.per_part; w += lanes) bad_heads[w] = 0u;
    __syncwarp();
    grid_dependency_wait();
    grid_launch_dependents();
    L l;
    l.init(p, lane);
    l.weights(t.w);
    DsqPair gw[L::P];
#pragma unroll
    for (int i = 0; i < L::P; ++i) gw[i] = 0ull;

    // Item by item (a part of a token's heads): where the loads are, and where the work is.
    const int64_t item = ((int64_t)block * BLOCK + threadIdx.x) / per_item;
    const int64_t lowest = ((int64_t)block * BLOCK + (threadIdx.x & ~31)) / per_item;         // of the warp
    const int64_t rounds = lowest < items ? (items - lowest + step - 1) / step : 0;
    struct At { int64_t item, token; int begin, head, last; };
    auto start = [&](At &a, int64_t i) {
        a.item = i;
        a.token = t.parts == 1 ? i : i / t.parts;
        a.begin = t.parts == 1 ? 0 : (int)(i - a.token * t.parts) * t.per_part;
        a.head = a.begin + of_warp;
        a.last = i < items ? min(a.begin + t.per_part, t.heads) : a.begin;
    };
    At in, at;
    const int turns = (t.per_part + by - 1) / by;              // of an item
    int left = turns;
    start(in, item);
    at = in;
    const T *gy, *x;
    T *y;
    auto from = [&]() {
        gy = (const T *)t.gy + in.token * t.g_token + in.head * t.g_head;
        x = (const T *)t.x + in.token * t.x_token + in.head * t.x_head;
    };
    auto to = [&]() { y = (T *)t.y + at.token * t.y_token + at.head * t.y_head; };
    from();
    to();
    Raw<T, VEC> next_x[U][2], next_g[U][2];
    auto load = [&]() {
        const bool on = in.head < in.last;
        l.load(gy, on, next_g);
        l.load(x, p.norm && on, next_x);
        in.head += by;
        if (--left == 0) {
            left = turns;
            start(in, in.item + step);
            from();
        } else {
            gy += by * t.g_head;
            x += by * t.x_head;
        }
    };
    load();
    for (int64_t round = 0; round < rounds; ++round) {
        if (WARP || at.head < at.last) l.template turns<WARP>(p, at.item < items ? at.token : 0, lane);
        bool any = false;
        for (int i = 0; i < turns; ++i) {
            DsqPair g[L::P], v[L::P];
            L::values(next_g, g);
            L::values(next_x, v);
            load();
            bool on = at.head < at.last;
            if (on) l.template turn<true>(g);
            if (p.norm) {
                DsqPair sum2 = 0ull, dot2 = 0ull;
#pragma unroll
                for (int k = 0; k < L::P; ++k) {
                    sum2 = dsq_pair_fma(v[k], v[k], sum2);
                    dot2 = dsq_pair_fma(dsq_pair_mul(g[k], l.w[k]), v[k], dot2);
                }
                const float sum = lanes_sum<L_>(sum_of(sum2), lanes), dot = lanes_sum<L_>(sum_of(dot2), lanes);
                const float mean = __fmaf_rn(sum, p.inv_d, p.eps), rstd = rsqrtf(mean);
                const float c = dot * rstd * p.inv_d;
                const bool bad = on && !in_range(mean, c);
                if (bad) {
                    if (lane == 0) bad_heads[(at.head - at.begin) >> 5] |= 1u << ((at.head - at.begin) & 31);
                    any = true;
                    on = false;
                }
                if (on) {
                    const DsqPair r = dsq_pair_of(rstd, rstd), less = dsq_pair_of(-c, -c);
#pragma unroll
                    for (int k = 0; k < L::P; ++k) {
                        const DsqPair m = dsq_pair_mul(v[k], r);
                        gw[k] = dsq_pair_fma(g[k], m, gw[k]);
                        g[k] = dsq_pair_mul(r, dsq_pair_fma(m, less, dsq_pair_mul(g[k], l.w[k])));
                    }
                }
            }
            if (on) l.store(y, g);
            at.head += by;
            y += by * t.y_head;
        }
        if (__any_sync(~0u, any)) wide_heads<T, true>(p, t, marks, lanes, t.per_part, at.token, at.begin, INTER, mine);
        start(at, at.item + step);
        to();
    }
    if (!t.part) return;
    // the block's sums: over the teams of a warp, then the warps, in one order
    __syncwarp();
#pragma unroll
    for (int i = 0; i < L::N; ++i) {
        float half[2];
        dsq_halves(gw[i / 2], half[0], half[1]);
        float s = half[i % 2];
        for (int o = 16; o >= lanes; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
        const Unit &u = l.unit[i / (2 * VEC)];
        const bool b = i / VEC % 2;
        if ((threadIdx.x & 31) < lanes && (b ? u.has_b : u.has_a)) mine[(b ? u.b : u.a) + i % VEC] += s;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < p.D; c += BLOCK) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < BLOCK / 32; ++w) s += sums[w][c];
        t.part[(int64_t)block * p.D + c] = s;
    }
}

// grad_w[c] = sum over the blocks of their sums, in one order, of q (blockIdx.y = 0) or k: 128 threads a column, eight
// columns, four loads of a thread on their way together
struct SumParams {
    const float *part[2];
    float *out[2];
    int blocks[2], D;
};
constexpr int SUM_COLS = 8, SUM_ROWS = 128;
__global__ void __launch_bounds__(SUM_COLS * SUM_ROWS) heads_sum_kernel(const SumParams p)
{
    __shared__ float s[SUM_ROWS / 4][SUM_COLS + 1];
    const int x = threadIdx.x % SUM_COLS, y = threadIdx.x / SUM_COLS, col = blockIdx.x * SUM_COLS + x;
    const float *part = p.part[blockIdx.y];
    const int rows = p.blocks[blockIdx.y];
    grid_dependency_wait();
    grid_launch_dependents();
    if (!p.out[blockIdx.y]) return;
    float a = 0.f;
    if (col < p.D)
        for (int r = y; r < rows; r += 4 * SUM_ROWS) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = r + SUM_ROWS * i < rows ? __ldcg(part + (int64_t)(r + SUM_ROWS * i) * p.D + col) : 0.f;
            a += (v[0] + v[1]) + (v[2] + v[3]);
        }
    // (a warp has four rows of the eight columns)
    a += __shfl_xor_sync(~0u, a, 8);
    a += __shfl_xor_sync(~0u, a, 16);
    if ((threadIdx.x & 31) < SUM_COLS) s[threadIdx.x >> 5][x] = a;
    __syncthreads();
    if (threadIdx.x >= 32 * SUM_COLS) return;
    const int c = threadIdx.x >> 5;
    a = s[threadIdx.x & 31][c];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a += __shfl_xor_sync(~0u, a, o);
    if ((threadIdx.x & 31) == 0 && blockIdx.x * SUM_COLS + c < p.D) p.out[blockIdx.y][blockIdx.x * SUM_COLS + c] = a;
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

// Parts of a token's heads.  `resident` takers of parts go round together, as often as there are parts for them, and a
// part costs its turns (as much as three heads, less than two where a warp shares them) and its heads, `by`
// at a time: the cheapest.
// Marks have room for MARKS words a block.
void set_parts(Tensor &t, int64_t tokens, int heads, int64_t resident, int by, int per_block)
{
    int64_t best = -1;
    const int most = heads < 64 ? heads : 64;
    for (int parts = 1; parts <= most; ++parts) {
        const int per_part = (heads + parts - 1) / parts;
        if (per_part > MARKS / per_block * 32) continue;
        const int64_t rounds = (tokens * parts + resident - 1) / resident, cost = rounds * ((by > 1 ? 2 : 3) + (per_part + by - 1) / by);
        if (best >= 0 && cost >= best) continue;
        best = cost;
        t.per_part = per_part;
    }
    t.parts = (heads + t.per_part - 1) / t.per_part;
}

template <class T, int VEC, int U, bool INTER, int L, bool BACK> int launch(Params &p, cudaStream_t s)
{
    const int pdl = dsq_launch_hooks().pdl;
    const int64_t sms = dsq_sm_count() > 0 ? dsq_sm_count() : 148, per_block = BLOCK / p.lanes;
    if constexpr (!BACK) {
        // heads enough for the teams of a warp to share a token's (a lane has more units just where 32 are too few)
        constexpr bool TEAMS = VEC == 1 ? U <= 2 : U == 1;
        const int heads = p.t[0].heads + p.t[1].heads;
        const bool warp = TEAMS && p.lanes < 32 && heads >= 2 * (32 / p.lanes);
        const int64_t items = warp ? BLOCK / 32 : per_block;
        set_parts(p.t[0], p.tokens, heads, sms * 5 * items, warp ? 32 / p.lanes : 1, (int)per_block);
        const int64_t blocks = (p.tokens * p.t[0].parts + items - 1) / items;
        if (blocks > 0x7FFFFFFF) return DSQ_ERR_SIZE;
        const auto kernel = warp ? heads_fwd_kernel<T, VEC, U, INTER, L, TEAMS> : heads_fwd_kernel<T, VEC, U, INTER, L, false>;
        return dsq_launch(kernel, dim3((unsigned)blocks), dim3(BLOCK), 0, s, pdl, 0, p);
    } else {
        // what is resident together, shared among q and k as their tokens' costs are (set_parts)
        const int64_t most = sms * (2 * U * VEC > 16 ? 2 : BACK_BLOCKS);
        int64_t blocks[2] = {0, 0};
        // (where not all units are turned a warp's sharing gains nothing: 8192 tokens of 8 + 8 heads of 96, half of each
        // turned, 36.8 us with it, 31.1 without)
        const int teams = 32 / p.lanes;
        const bool warp = L && p.t[0].heads >= teams && (!p.t[1].heads || p.t[1].heads >= teams);
        const int64_t of_block = warp ? BLOCK / 32 : per_block;
        for (int i = 0; i < 2; ++i) {
            Tensor &t = p.t[i];
            if (!t.heads) continue;
            auto cost = [&](int heads) { return heads ? (warp ? 2 + (heads + teams - 1) / teams : 3 + heads) : 0; };
            int64_t share = most * cost(t.heads) / (cost(p.t[0].heads) + cost(p.t[1].heads));
            if (share < 1) share = 1;
            set_parts(t, p.tokens, t.heads, share * of_block, warp ? teams : 1, (int)per_block);
            const int64_t need = (p.tokens * t.parts + of_block - 1) / of_block;
            blocks[i] = need < share ? need : share;
        }
        p.q_blocks = (int)blocks[0];
        p.k_blocks = (int)blocks[1];
        if (p.t[1].part) p.t[1].part = p.t[0].part + blocks[0] * p.D;
        const auto kernel = warp ? heads_bwd_kernel<T, VEC, U, INTER, L, (L > 0)> : heads_bwd_kernel<T, VEC, U, INTER, L, false>;
        return dsq_launch(kernel, dim3((unsigned)(blocks[0] + blocks[1])), dim3(BLOCK), 0, s, pdl, 0, p);
    }
}

// Fills in what depends on the vectors' length and the units of a lane.
void set_lanes(Params &p, int vec, int per_lane)
{
    const int turned = p.R / (2 * vec), rest = (p.D - p.R + 2 * vec - 1) / (2 * vec);
    p.units = turned + rest;
    p.lanes = 1;
    while (p.lanes * per_lane < p.units && p.lanes < 32) p.lanes *= 2;
}

// One unit a lane, or as many as 32 lanes need.
template <class T, bool INTER, bool BACK> int pick(Params &p, bool vectors, cudaStream_t s)
{
    constexpr int V = vec_of<T>(), U = 1;
    if (!vectors) {
        set_lanes(p, 1, 1);
        return p.units <= 64 ? launch<T, 1, 2, INTER, 0, BACK>(p, s) : launch<T, 1, 8, INTER, 0, BACK>(p, s);
    }
    set_lanes(p, V, U);
    if (p.R == p.D && p.lanes * U == p.units) {
        if (p.lanes == 16 / U) return launch<T, V, U, INTER, 16 / U, BACK>(p, s);
        if (p.lanes == 8 / U) return launch<T, V, U, INTER, 8 / U, BACK>(p, s);
        if (p.lanes == 4 / U) return launch<T, V, U, INTER, 4 / U, BACK>(p, s);
    }
    if constexpr (V == 4) {
        if (p.units > 32) return launch<T, V, 2, INTER, 0, BACK>(p, s);
    }
    return launch<T, V, U, INTER, 0, BACK>(p, s);
}

template <bool BACK> int start(Params &p, bool vectors, bool inter, int dtype, cudaStream_t s)
{
    switch (dtype) {
    case DSQ_F32: return inter ? pick<float, true, BACK>(p, vectors, s) : pick<float, false, BACK>(p, vectors, s);
    case DSQ_BF16: return inter ? pick<__nv_bfloat16, true, BACK>(p, vectors, s) : pick<__nv_bfloat16, false, BACK>(p, vectors, s);
    default: return inter ? pick<__half, true, BACK>(p, vectors, s) : pick<__half, false, BACK>(p, vectors, s);
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
        if (!apart(tokens, h->heads, h->y_token, h->y_head, p.D) || (i && h->y == q->y)) return DSQ_ERR_SHAPE;
        Tensor &t = p.t[i];
        t.x = h->x; t.y = h->y; t.w = h->weight;
        t.x_token = h->x_token; t.x_head = h->x_head; t.y_token = h->y_token; t.y_head = h->y_head;
        t.heads = (int)h->heads;
        vectors = vectors && in_vectors(h->x, h->x_token, h->x_head, vec, size) &&
                  in_vectors(h->y, h->y_token, h->y_head, vec, size);
    }
    return start<false>(p, vectors, rotary->interleaved != 0, dtype, (cudaStream_t)stream);
}

size_t dsq_headnorm_bwd_workspace_bytes(int64_t head_dim)
{
    if (head_dim <= 0 || head_dim > MAX_DIM) return DSQ_WS_BYTES;
    const int sms = dsq_sm_count() > 0 ? dsq_sm_count() : 148;
    return DSQ_WS_BYTES + (size_t)(sms * BACK_BLOCKS + 2) * (size_t)head_dim * 4;
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
        if (!apart(tokens, h->heads, h->gx_token, h->gx_head, p.D) || (i && h->grad_x == q->grad_x)) return DSQ_ERR_SHAPE;
        Tensor &t = p.t[i];
        t.gy = h->grad_y; t.x = h->x; t.y = h->grad_x; t.w = h->weight;
        t.g_token = h->gy_token; t.g_head = h->gy_head;
        t.x_token = h->x_token; t.x_head = h->x_head; t.y_token = h->gx_token; t.y_head = h->gx_head;
        t.heads = (int)h->heads;
        // (sums of both are made where either is wanted)
        t.part = sums ? (float *)((char *)workspace + DSQ_WS_BYTES) : nullptr;
        sp.out[i] = h->grad_weight;
        vectors = vectors && in_vectors(h->grad_y, h->gy_token, h->gy_head, vec, size) &&
                  in_vectors(h->grad_x, h->gx_token, h->gx_head, vec, size) &&
                  (!norm || in_vectors(h->x, h->x_token, h->x_head, vec, size));
    }
    if (sums && !dsq_aligned16(workspace)) return DSQ_ERR_ALIGN;
    if (sums && ws_bytes < dsq_headnorm_bwd_workspace_bytes(p.D)) return DSQ_ERR_SIZE;
    st = start<true>(p, vectors, rotary->interleaved != 0, dtype, (cudaStream_t)stream);
    if (st || !sums) return st;
    for (int i = 0; i < 2; ++i) sp.part[i] = p.t[i].part;
    sp.blocks[0] = p.q_blocks; sp.blocks[1] = p.k_blocks;
    sp.D = p.D;
    return dsq_launch(heads_sum_kernel, dim3((unsigned)((p.D + SUM_COLS - 1) / SUM_COLS), 2), dim3(SUM_COLS * SUM_ROWS), 0, (cudaStream_t)stream,
                      dsq_launch_hooks().pdl, 0, sp);
}

}  // extern "C"
