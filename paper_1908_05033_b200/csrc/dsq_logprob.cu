// Log probabilities of given tokens with entropy and the most probable alternatives of rows of
// logits, and the logits' gradient (what stands behind a decoder's last product).
//
//   z = scale x,  lse = m + log s,  s = sum e^(z - m),  logp = z_t - lse,
//   H = log s - t / s,  t = sum (z - m) e^(z - m)
//   grad_j = scale (g ([j = t] - p_j) - g_H p_j (log p_j + H)),  p = e^(z - lse)
//
// HBM-bound: the forward kernel reads the logits once, the backward one reads and writes them once.
//   * Forward: a row goes to a block or, where there are few, to a cluster of up to eight, whose first
//     block joins the parts.  A thread keeps m, s and t of its elements in one pass; four vectors are
//     on their way together.  The exponents are powers of two, x c - M with c = scale log2 e and M = m c as
//     binary32 rounds it: one fused operation, the rounding of M being the same in s, t and the target's
//     exponent.  Four instructions an element for the three; where an element is -infinity, or M is large enough for its
//     rounding to matter, (x - m) c instead, held above -1000 (six).
//   * Alternatives: a thread leaves the largest element of each turn of its loop in shared memory.  Fours of
//     threads form groups; the top-th of the groups' largest elements bounds from below what can be among the
//     first `top`, and only turns whose largest is above the bound are read again (from L2), by as many threads as
//     they have vectors; what passes goes to shared memory, where ranks are counted.  Order and ties are those of
//     (value, lowest index), as one 64-bit key.  Where the bound is the value of most elements (a mask that leaves fewer groups than
//     `top` anything) the elements above it are collected alone and its lowest indices fill up behind them, in a scan that ends
//     with the turn that has enough: 2048 rows of 128000 bf16 with three left, 20 alternatives, 152 us (111 without a
//     mask; the largest `top` times one after the other 3790).  That is left for rows whose large elements are many,
//     different and all with the same few threads.
//   4096 rows of 128000 bf16 with five alternatives: 222 us, 4.7 TB/s (197 where the same rows come again and L2 has some of
//   them): nothing is saturated (issue slots 63 %, DRAM 53 %), blocks between their passes and a last wave that is not
//   full; without alternatives 161.  Fewer rows more so: 1024 57 us, 300 32, 75 to 148 13.5.  One row: 9.6 us, a chain of a
//   load, three barriers, a second load of a few vectors and the cluster's exchange.
//   * Backwards: a block takes a piece of a row, reads it and writes it.  2048 rows of 128000 bf16: 175 us, 6.0 TB/s (158 where
//   the same rows come again: L2).
#include "dsq_launch.h"
#include "dsq_pairs.cuh"
#include "dsq_ptx.cuh"
#include "dsq_types.cuh"

using namespace dsq_ptx;

namespace {

constexpr int MAX_TOP = 32, MAX_CLUSTER = 8, AHEAD = 4, SHARE = 4;      // SHARE: threads of a group
constexpr int ROOM = 1088;        // of candidates: 128 threads' vectors where fewer groups than `top` have any
constexpr int SLOTS = 16, HITS = 512;      // turns that are told apart, and how many may be read again
constexpr float LOWEST = -3.402823466e38f, LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
// 2^x of what is lower is zero
constexpr float NOTHING = -1000.f;
// times log2 e it is finite
constexpr float MAX_SCALE = 0x1p127f;
// M is taken below this: its rounding is at most 2^-8 then
constexpr float FAR = 65536.f;

struct FwdParams {
    const void *x;
    const int64_t *targets;
    float *logp, *entropy, *lse, *top_logp;
    int64_t *top_ids;
    int64_t ld;
    int V, top, cluster;
    float scale;
};

struct BwdParams {
    const void *x;
    const int64_t *targets;
    const float *lse, *entropy, *g_logp, *g_entropy;
    void *grad;
    int64_t ld, grad_ld;
    int V, segments;
    float scale;
};

__device__ __forceinline__ float ex2(float v)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// (a NaN stays one)
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
template <class T> constexpr int vec_of() { return 16 / (int)sizeof(T); }

__device__ __forceinline__ uint4 load_16(const void *p)
{
    uint4 r;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}
template <class T> __device__ __forceinline__ void values(const uint4 &r, float (&f)[vec_of<T>()])
{
    if constexpr (sizeof(T) == 4) {
        f[0] = __uint_as_float(r.x); f[1] = __uint_as_float(r.y);
        f[2] = __uint_as_float(r.z); f[3] = __uint_as_float(r.w);
    } else {
        DsqRaw8<T> raw;
        raw.v[0] = r;
        dsq_unpack8(raw, f);
    }
}
// -infinity in every place
template <class T> __device__ __forceinline__ uint4 nothing()
{
    const uint32_t w = sizeof(T) == 4 ? 0xFF800000u : std::is_same<T, __half>::value ? 0xFC00FC00u : 0xFF80FF80u;
    return make_uint4(w, w, w, w);
}
// the largest element, NaN left out (of nothing but NaN: NaN)
template <class T> __device__ __forceinline__ float largest(const uint4 (&r)[AHEAD])
{
    if constexpr (sizeof(T) == 4) {
        float m = __uint_as_float(r[0].x);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            m = fmaxf(fmaxf(fmaxf(m, __uint_as_float(r[i].x)), __uint_as_float(r[i].y)),
                      fmaxf(__uint_as_float(r[i].z), __uint_as_float(r[i].w)));
        return m;
    } else {
        typedef typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type T2;
        const T2 *v = reinterpret_cast<const T2 *>(r);
        T2 m = v[0];
#pragma unroll
        for (int i = 1; i < 4 * AHEAD; ++i) m = __hmax2(m, v[i]);
        return fmaxf(dsq_to_f32(m.x), dsq_to_f32(m.y));
    }
}

// Key of an element: by value, equal ones by index, the lowest first; NaN below all, nothing at all 0.
__device__ __forceinline__ unsigned long long key_of(float v, int index)
{
    const uint32_t u = __float_as_uint(v + 0.f);              // (-0 is 0)
    uint32_t k = (int)u < 0 ? ~u : u | 0x80000000u;
    if (v != v) k = 0u;
    return (unsigned long long)k << 32 | (uint32_t)~index;
}
__device__ __forceinline__ float value_of(unsigned long long key)
{
    const uint32_t k = (uint32_t)(key >> 32);
    if (k == 0u) return __uint_as_float(0x7FC00000u);
    return __uint_as_float((int)k < 0 ? k & 0x7FFFFFFFu : ~k);
}
__device__ __forceinline__ int index_of(unsigned long long key) { return (int)~(uint32_t)key; }

// Sums of powers of two: s of 2^d, t of d 2^d, d = x c - M with M = m c rounded; where that is far, d = (x - m) c.
// Sums are joined on the larger m.
struct Sums { float m, s, t; };
// what d of m' is less beside m: m' c - m c, each product as it is taken
__device__ __forceinline__ float between(float from, float to, float c)
{
    const float F = from * c, T = to * c;
    const bool f = fabsf(F) < FAR, t = fabsf(T) < FAR;
    return max_nan(f ? (t ? F - T : __fmaf_rn(-to, c, F)) : t ? __fmaf_rn(from, c, -T) : (from - to) * c, NOTHING);
}
// the exponent of x beside m
__device__ __forceinline__ float exponent(float x, float m, float c)
{
    const float M = m * c;
    return max_nan(fabsf(M) < FAR ? __fmaf_rn(x, c, -M) : (x - m) * c, NOTHING);
}
__device__ __forceinline__ void move_to(Sums &v, float m, float c)
{
    const float d = between(v.m, m, c), e = ex2(d);
    v.t = __fmaf_rn(v.s, d, v.t) * e;
    v.s *= e;
    v.m = m;
}
// of the lanes of a warp, the same in all
__device__ __forceinline__ Sums joined(Sums v, float c)
{
    float m = v.m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
    move_to(v, m, c);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        v.s += __shfl_xor_sync(~0u, v.s, o);
        v.t += __shfl_xor_sync(~0u, v.t, o);
    }
    return v;
}

// Where a row's whole vectors lie: `head` single elements, nv vectors, `tail` single ones.
template <class T> struct Cut {
    const T *row;
    int head, nv, tail;
    __device__ __forceinline__ Cut(const T *r, int V) : row(r)
    {
        head = min(V, (int)((16 - (reinterpret_cast<uintptr_t>(r) & 15)) & 15) / (int)sizeof(T));
        nv = (V - head) / vec_of<T>();
        tail = V - head - nv * vec_of<T>();
    }
    __device__ __forceinline__ int index(int v) const { return head + v * vec_of<T>(); }
    __device__ __forceinline__ int single(int i) const { return i < head ? i : i + nv * vec_of<T>(); }
};

// Ranks of n keys, all different: f(rank, key) for each, by one lane of the warp that counts.
template <int THREADS, class F> __device__ __forceinline__ void ranked(const unsigned long long *keys, int n, F f)
{
    const int lane = threadIdx.x & 31;
    for (int i = threadIdx.x >> 5; i < n; i += THREADS / 32) {
        const unsigned long long mine = keys[i];
        int rank = 0;
        for (int j = 0; j < n; j += 32) rank += __popc(__ballot_sync(~0u, j + lane < n && keys[j + lane] > mine));
        if (lane == 0) f(rank, mine);
    }
}

__device__ __forceinline__ void st_cluster_64(uint32_t addr, unsigned long long v)
{
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}

// What a block has of a row for its alternatives.
template <class T> struct Part {
    Cut<T> cut;
    int v0, v1, singles;              // its vectors, how many single elements
    int turns, per_slot;
    const float *slot_most;
    uint32_t *hit;
    unsigned long long *found;
    int *hits, *count;
};

// The vectors of the turns whose largest element passes, f(element, index) for each, a thread a vector; f(...) for the single ones
// too.  False where there are more turns than there is room for.  (*hits and *count are 0, and every thread knows.)
template <class T, int THREADS, class P, class F>
__device__ __forceinline__ bool look_again(const Part<T> &a, P passes, F f)
{
    constexpr int VEC = vec_of<T>();
    const int tid = threadIdx.x;
    if (tid < a.singles) f(dsq_to_f32(a.cut.row[a.cut.single(tid)]), a.cut.single(tid));
    for (int i = 0; i * a.per_slot < a.turns; ++i) {
        if (a.v0 + i * a.per_slot * AHEAD * THREADS + tid >= a.v1) break;
        if (!passes(a.slot_most[i * THREADS + tid])) continue;
        const int at = atomicAdd(a.hits, 1);
        if (at < HITS) a.hit[at] = (uint32_t)tid | (uint32_t)i << 16;
    }
    __syncthreads();
    const int per_hit = a.per_slot * AHEAD, n_hits = *a.hits;
    if (n_hits > HITS) return false;
    for (int64_t w = tid; w < (int64_t)n_hits * per_hit; w += THREADS) {
        const int h = (int)(w / per_hit), k = (int)(w - (int64_t)h * per_hit);
        const int64_t v = a.v0 + ((int64_t)(a.hit[h] >> 16) * per_hit + k) * THREADS + (a.hit[h] & 0xFFFFu);
        if (v >= a.v1) continue;
        float e[VEC];
        values<T>(load_16(a.cut.row + a.cut.head + v * VEC), e);
#pragma unroll
        for (int i = 0; i < VEC; ++i) f(e[i], a.cut.index((int)v) + i);
    }
    return true;
}

// The first `top` where most elements are equal to the bound (a mask's value; a row of one value): those above it, of
// which there are fewer, and behind them the lowest indices of equal ones, in one scan that ends with the turn that has enough.
// `masked`: the bound is LOWEST or below, and behind LOWEST come -infinity and NaN.  *count: of the candidates in `found`,
// beyond ROOM where there is no room for those above.
template <class T, int THREADS> __device__ __forceinline__ void take_equal(const Part<T> &a, int top, float least, bool masked)
{
    constexpr int VEC = vec_of<T>();
    const int tid = threadIdx.x, lane = tid & 31;
    const float none = __uint_as_float(0xFF800000u);
    if (masked) {
        // (a slot's largest tells whether LOWEST is a mask; single ones of it between larger elements are found with these)
        bool low = false;
        for (int i = 0; i * a.per_slot < a.turns; ++i) {
            if (a.v0 + i * a.per_slot * AHEAD * THREADS + tid >= a.v1) break;
            low = low || a.slot_most[i * THREADS + tid] == LOWEST;
        }
        least = __syncthreads_or(low) ? LOWEST : none;
    }
    __syncthreads();                                           // (*hits and *count have been read)
    if (tid == 0) *a.hits = *a.count = 0;
    __syncthreads();
    auto add = [&](float v, int index) {
        const int at = atomicAdd(a.count, 1);
        if (at < ROOM) a.found[at] = key_of(v, index);
    };
    const bool room = look_again<T, THREADS>(a, [&](float most) { return most > least; }, [&](float v, int index) {
        if (v > least) add(v, index);
    });
    __syncthreads();
    if (!room) {
        if (tid == 0) *a.count = ROOM + 1;
        __syncthreads();
        return;
    }
    int have = *a.count;
    for (;;) {                                                 // least: NaN in the end
        __syncthreads();                                       // (everybody has read *count)
        if (have >= top) return;
        auto equal = [&](float v) { return least != least ? v != v : v == least; };
        auto single = [&](int from, int to) {
            if (tid >= from && tid < to) {
                const float v = dsq_to_f32(a.cut.row[a.cut.single(tid)]);
                if (equal(v)) add(v, a.cut.single(tid));
            }
            __syncthreads();
            have = *a.count;
            __syncthreads();
        };
        if (a.singles > 0) single(0, a.cut.head);
        for (int v0 = a.v0; v0 < a.v1 && have < top; v0 += THREADS) {
            float e[VEC];
            uint32_t mine = 0u;
            if (v0 + tid < a.v1) {
                values<T>(load_16(a.cut.row + a.cut.head + (int64_t)(v0 + tid) * VEC), e);
#pragma unroll
                for (int i = 0; i < VEC; ++i) mine |= equal(e[i]) ? 1u << i : 0u;
            }
            // the warp's first ones, as many as are still wanted
            int before = __popc(mine);
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(~0u, before, o);
                if (lane >= o) before += v;
            }
            const int wanted = min(__shfl_sync(~0u, before, 31), top - have);
            before -= __popc(mine);
            int at = 0;
            if (lane == 0 && wanted > 0) at = atomicAdd(a.count, wanted);
            at = __shfl_sync(~0u, at, 0);
            for (; mine && before < wanted; mine &= mine - 1, ++before)
                a.found[at + before] = key_of(least, a.cut.index(v0 + tid) + __ffs(mine) - 1);
            __syncthreads();
            have = *a.count;
            __syncthreads();
        }
        if (a.singles > 0 && have < top) single(a.cut.head, a.singles);
        if (!masked || least != least) return;
        least = least == LOWEST ? none : __uint_as_float(0x7FC00000u);
    }
}

template <class T, bool TOP, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) logprob_fwd_kernel(const __grid_constant__ FwdParams p)
{
    constexpr int VEC = vec_of<T>(), GROUPS = THREADS / SHARE;
    static_assert(GROUPS >= MAX_TOP, "a group for each of the first");
    __shared__ Sums warp_sums[THREADS / 32];
    __shared__ Sums block_sums[MAX_CLUSTER];
    __shared__ unsigned long long lists[TOP ? MAX_CLUSTER * MAX_TOP : 1];      // of the first block: all blocks' first `top`
    __shared__ unsigned long long bests[TOP ? GROUPS : 1], found[TOP ? ROOM : 1], bound_key;
    __shared__ float slot_most[TOP ? SLOTS * THREADS : 1];
    __shared__ uint32_t hit[TOP ? HITS : 1];                   // thread, slot
    __shared__ int count, hits;
    const int rank = p.cluster > 1 ? (int)cluster_ctarank() : 0;
    const int64_t row = blockIdx.x / p.cluster;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    grid_dependency_wait();
    grid_launch_dependents();
    // (the first block's shared memory is written from the others once it has started)
    if (p.cluster > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const Cut<T> cut((const T *)p.x + row * p.ld, p.V);
    const int v0 = (int)((int64_t)cut.nv * rank / p.cluster), v1 = (int)((int64_t)cut.nv * (rank + 1) / p.cluster);
    const int singles = rank == 0 ? cut.head + cut.tail : 0;
    const float c = p.scale * LOG2E;
    const T *vecs = cut.row + cut.head;
    float wanted = 0.f;                                        // the target's logit
    int64_t target = -1;
    if (rank == 0 && tid == 0 && p.logp) {
        target = p.targets[row];
        if (target >= 0 && target < p.V) wanted = dsq_to_f32(cut.row[target]);
    }

    // one pass: m, s, t of this thread's elements, and in which turn m came
    const T *at = vecs + ((int64_t)v0 + tid) * VEC;            // of the next turn
    auto load = [&](uint4 (&r)[AHEAD]) {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) r[j] = load_16(at + j * THREADS * VEC);
        at += AHEAD * THREADS * VEC;
    };
    const int turns = (v1 - v0 + THREADS * AHEAD - 1) / (THREADS * AHEAD), full = (v1 - v0) / (THREADS * AHEAD);
    float m = LOWEST;
    int best_turn = -1;
    DsqPair s2 = 0ull, t2 = 0ull;
    const DsqPair c2 = dsq_pair_of(c, c);
    // (x - m) c above NOTHING: any element
    auto any_vector = [&](const uint4 &r) {
        const bool near = fabsf(m * c) < FAR;
        const DsqPair less = dsq_pair_of(-m, -m), lessM = dsq_pair_of(-(m * c), -(m * c));
        float f[VEC];
        values<T>(r, f);
#pragma unroll
        for (int i = 0; i < VEC; i += 2) {
            const DsqPair x = dsq_pair_of(f[i], f[i + 1]);
            const DsqPair d = near ? dsq_pair_fma(x, c2, lessM) : dsq_pair_mul(dsq_pair_add(x, less), c2);
            float d0, d1;
            dsq_halves(d, d0, d1);
            d0 = max_nan(d0, NOTHING);
            d1 = max_nan(d1, NOTHING);
            const DsqPair e = dsq_pair_of(ex2(d0), ex2(d1));
            s2 = dsq_pair_add(s2, e);
            t2 = dsq_pair_fma(dsq_pair_of(d0, d1), e, t2);
        }
    };
    // m of all so far
    auto raise = [&](float most, int turn) {
        if (!(most > m)) return;
        const float d = between(m, most, c), e = ex2(d);
        const DsqPair e2 = dsq_pair_of(e, e);
        t2 = dsq_pair_mul(dsq_pair_fma(s2, dsq_pair_of(d, d), t2), e2);
        s2 = dsq_pair_mul(s2, e2);
        m = most;
        best_turn = turn;
    };
    if (TOP && v0 + tid < v1) best_turn = 0;                   // (where m stays LOWEST: the first turn)
    bool general = false;                                      // elements of -infinity have been seen
    // a slot's turns, its largest element so far
    const int per_slot = (turns + SLOTS - 1) / SLOTS;
    int slot = 0, in_slot = 0;
    float so_far = 0.f;
    auto note = [&](float most) {
        if (!TOP) return;
        so_far = in_slot == 0 ? most : fmaxf(so_far, most);
        slot_most[slot * THREADS + tid] = so_far;
        if (++in_slot == per_slot) {
            in_slot = 0;
            ++slot;
        }
    };
    uint4 next[AHEAD];
    // the last turn's vectors, as far as there are any
    auto load_rest = [&]() {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            next[j] = v0 + (full * AHEAD + j) * THREADS + tid < v1 ? load_16(at + j * THREADS * VEC) : nothing<T>();
    };
    if (full > 0) load(next);
    else load_rest();
#pragma unroll 1
    for (int turn = 0; turn < full; ++turn) {
        uint4 r[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) r[j] = next[j];
        if (turn + 1 < full) load(next);
        else load_rest();
        const float most = largest<T>(r);
        note(most);
        raise(most, turn);
        const float M = m * c;
        if (!general && fabsf(M) < FAR) {
            const DsqPair s0 = s2, t0 = t2, less = dsq_pair_of(-M, -M);
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                float f[VEC];
                values<T>(r[j], f);
#pragma unroll
                for (int i = 0; i < VEC; i += 2) {
                    const DsqPair d = dsq_pair_fma(dsq_pair_of(f[i], f[i + 1]), c2, less);
                    float d0, d1;
                    dsq_halves(d, d0, d1);
                    const DsqPair e = dsq_pair_of(ex2(d0), ex2(d1));
                    s2 = dsq_pair_add(s2, e);
                    t2 = dsq_pair_fma(d, e, t2);
                }
            }
            float a, b;
            dsq_halves(t2, a, b);
            if (a + b == a + b) continue;
            // (-infinity times 0, or a NaN of the row's: once more)
            s2 = s0;
            t2 = t0;
            general = true;
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) any_vector(r[j]);
    }
    if (full < turns) {
        const float most = largest<T>(next);                   // (what is not there is -infinity)
        note(most);
        raise(most, full);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (v0 + (full * AHEAD + j) * THREADS + tid < v1) any_vector(next[j]);
    }
    Sums sum;
    {
        float a, b;
        dsq_halves(s2, a, b);
        sum.s = a + b;
        dsq_halves(t2, a, b);
        sum.t = a + b;
        sum.m = m;
    }
    if (tid < singles) {
        const float v = dsq_to_f32(cut.row[cut.single(tid)]);
        // (-infinity and NaN as in the loop: less LOWEST nothing, and NaN)
        const float one_m = fmaxf(v, LOWEST), d = exponent(v, one_m, c), e = ex2(d);
        Sums one = {one_m, e, d * e};
        const float both = fmaxf(sum.m, one_m);
        move_to(sum, both, c);
        move_to(one, both, c);
        sum.s += one.s;
        sum.t += one.t;
    }
    sum = joined(sum, c);
    if (lane == 0) warp_sums[warp] = sum;
    if (TOP) {
        if (tid == 0) {
            count = hits = 0;
            bound_key = 0ull;
        }
        // the largest of a group, its index no lower than it is
        unsigned long long best = 0ull;
        if (best_turn >= 0) {
            const int first = v0 + best_turn * AHEAD * THREADS + tid, last = first + min(AHEAD - 1, (v1 - 1 - first) / THREADS) * THREADS;
            // (m is LOWEST where all are -infinity, NaN or LOWEST: below them all, then, but above what is not there)
            best = m > LOWEST ? key_of(m, cut.index(last) + VEC - 1) : (unsigned long long)(uint32_t)~(cut.index(last) + VEC - 1);
        }
#pragma unroll
        for (int o = 1; o < SHARE; o <<= 1) {
            const unsigned long long other = __shfl_xor_sync(~0u, best, o);
            best = best > other ? best : other;
        }
        if (tid % SHARE == 0) bests[tid / SHARE] = best;
        __syncthreads();
        // the `top`-th of them
        {
            int above = 0;
#pragma unroll 4
            for (int j = tid % SHARE; j < GROUPS; j += SHARE) above += bests[j] > best;
#pragma unroll
            for (int o = 1; o < SHARE; o <<= 1) above += __shfl_xor_sync(~0u, above, o);
            if (tid % SHARE == 0 && above == p.top - 1 && best != 0ull) bound_key = best;
        }
        __syncthreads();
        const unsigned long long bound = bound_key;
        const Part<T> part = {cut, v0, v1, singles, turns, per_slot, slot_most, hit, found, &hits, &count};
        // turns that may have some, and their vectors, a thread each (no bound: all)
        const bool masked = bound != 0ull && bound >> 32 == 0ull;
        const float least = value_of(bound);
        bool room = false;
        if (!masked) {
            room = look_again<T, THREADS>(part, [&](float most) { return bound == 0ull || most >= least; }, [&](float v, int index) {
                const unsigned long long key = key_of(v, index);
                if (key < bound) return;
                const int at = atomicAdd(&count, 1);
                if (at < ROOM) found[at] = key;
            });
            __syncthreads();
            room = room && count <= ROOM;
        }
        if (!room && bound != 0ull) take_equal<T, THREADS>(part, p.top, least, masked);
        else if (!room && tid == 0) count = ROOM + 1;
    }
    __syncthreads();
    if (p.cluster > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (tid < 32) {
        const Sums nothing_yet = {LOWEST, 0.f, 0.f};
        const Sums all = joined(tid < THREADS / 32 ? warp_sums[tid] : nothing_yet, c);
        if (tid == 0) {
            if (p.cluster == 1) block_sums[0] = all;
            else {
                const uint32_t at = map_to_cta(smem_u32(&block_sums[rank]), 0);
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(all.m) : "memory");
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at + 4), "f"(all.s) : "memory");
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at + 8), "f"(all.t) : "memory");
            }
        }
    }
    if (TOP) {
        const uint32_t list = p.cluster == 1 ? smem_u32(lists) : map_to_cta(smem_u32(lists + rank * p.top), 0);
        auto put = [&](int at, unsigned long long key) {
            if (p.cluster == 1) lists[at] = key;
            else st_cluster_64(list + 8 * at, key);
        };
        const int n = count;
        // (fewer than `top`: the rest of the list is nothing)
        for (int i = tid; i < p.top; i += THREADS)
            if (i >= n) put(i, 0ull);
        if (n <= ROOM) {
            ranked<THREADS>(found, n, [&](int at, unsigned long long key) {
                if (at < p.top) put(at, key);
            });
        } else {
            // More than there is room for (many different large elements, and all with the same few threads): one after
            // the other, the largest below the one before.
            unsigned long long last = ~0ull;
            for (int i = 0; i < p.top; ++i) {
                unsigned long long best = 0ull;
                auto take = [&](float v, int index) {
                    const unsigned long long key = key_of(v, index);
                    if (key < last && key > best) best = key;
                };
                if (tid < singles) take(dsq_to_f32(cut.row[cut.single(tid)]), cut.single(tid));
#pragma unroll 1
                for (int v = v0 + tid; v < v1; v += THREADS) {
                    float f[VEC];
                    values<T>(load_16(vecs + (int64_t)v * VEC), f);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) take(f[e], cut.index(v) + e);
                }
                for (int o = 16; o > 0; o >>= 1) {
                    const unsigned long long other = __shfl_xor_sync(~0u, best, o);
                    best = best > other ? best : other;
                }
                __syncthreads();
                if (lane == 0) bests[warp] = best;
                __syncthreads();
                for (int w = 0; w < THREADS / 32; ++w) best = best > bests[w] ? best : bests[w];
                if (tid == 0) put(i, best);
                last = best;
            }
        }
    }
    if (p.cluster > 1) cluster_sync_all();
    else __syncthreads();
    if (rank != 0) return;
    const Sums nothing_yet = {LOWEST, 0.f, 0.f};
    const Sums all = joined(lane < p.cluster ? block_sums[lane] : nothing_yet, c);
    const float log_s = log2f(all.s);
    // (a row without any: everything is improbable, and there is nothing to be uncertain about)
    const bool empty = all.s == 0.f;
    const float none = __uint_as_float(0xFF800000u), nan = __uint_as_float(0x7FC00000u);
    auto logp_of = [&](float v) {
        const float M = all.m * c;
        if (empty) return none;
        return fabsf(M) < FAR && fabsf(v * c) < FAR ? (__fmaf_rn(v, c, -M) - log_s) * LN2 : (v - all.m) * p.scale - log_s * LN2;
    };
    if (tid == 0) {
        if (p.logp) p.logp[row] = target < 0 ? 0.f : target >= p.V ? nan : logp_of(wanted);
        if (p.entropy) {
            const float h = (log_s - all.t / all.s) * LN2;
            p.entropy[row] = empty || h < 0.f ? 0.f : h;
        }
        if (p.lse) {
            const float M = all.m * c;
            p.lse[row] = empty ? none : fabsf(M) < FAR ? __fmaf_rn(M, LN2, log_s * LN2) : __fmaf_rn(all.m, p.scale, log_s * LN2);
        }
    }
    if (TOP)
        ranked<THREADS>(lists, p.cluster * p.top, [&](int at, unsigned long long key) {
            if (at >= p.top || key == 0ull) return;
            if (p.top_ids) p.top_ids[row * p.top + at] = index_of(key);
            if (p.top_logp) p.top_logp[row * p.top + at] = logp_of(value_of(key));
        });
}

constexpr int BWD_THREADS = 256, BWD_AHEAD = 2;
template <class T> constexpr int bwd_segment() { return BWD_THREADS * BWD_AHEAD * vec_of<T>() * 4; }   // elements, four turns

// SAME: logits and gradients lie alike in their vectors
template <class T, bool SAME>
__global__ void __launch_bounds__(BWD_THREADS) logprob_bwd_kernel(const __grid_constant__ BwdParams p)
{
    constexpr int VEC = vec_of<T>();
    const int64_t row = blockIdx.x / p.segments;
    const int segment = (int)(blockIdx.x - row * p.segments);
    grid_dependency_wait();
    grid_launch_dependents();
    const T *x = (const T *)p.x + row * p.ld;
    T *grad = (T *)p.grad + row * p.grad_ld;
    const int64_t target = p.targets ? p.targets[row] : -1;
    float g = p.g_logp && target >= 0 ? p.g_logp[row] : 0.f;
    const float ge = p.g_entropy ? p.g_entropy[row] : 0.f;
    if (g != 0.f && target >= p.V) g = __uint_as_float(0x7FC00000u);
    const float lse = p.lse[row], h = p.entropy ? p.entropy[row] : 0.f;
    // rows that nothing comes back to, and rows without any probability
    const int at_target = target >= 0 && target < p.V ? (int)target : -1;
    const bool zero = (g == 0.f && ge == 0.f) || lse == __uint_as_float(0xFF800000u);
    const float a = g * p.scale, b = ge * p.scale;
    // -p (a + b (log p + H)) of z = scale x
    auto of = [&](float v) {
        const float l = __fmaf_rn(v, p.scale, -lse), l2 = max_nan(l * LOG2E, NOTHING);
        return -(ex2(l2) * __fmaf_rn(b, max_nan(l, NOTHING) + h, a));
    };
    auto one = [&](int i) {
        float v = 0.f;
        if (!zero) {
            v = of(dsq_to_f32(x[i]));
            if (i == at_target) v += a;
        }
        grad[i] = dsq_from_f32<T>(v);
    };
    if constexpr (!SAME) {
        const int from = segment * bwd_segment<T>(), to = min(p.V, from + bwd_segment<T>());
        for (int i = from + threadIdx.x; i < to; i += BWD_THREADS) one(i);
    } else {
        const Cut<T> cut(x, p.V);
        if (segment == 0 && threadIdx.x < cut.head + cut.tail) one(cut.single(threadIdx.x));
        constexpr int PER = bwd_segment<T>() / VEC;
        const int from = segment * PER, to = min(cut.nv, from + PER);
        const T *xv = x + cut.head;
        T *gv = grad + cut.head;
#pragma unroll 1
        for (int v0 = from + threadIdx.x; v0 < to; v0 += BWD_THREADS * BWD_AHEAD) {
            uint4 r[BWD_AHEAD];
#pragma unroll
            for (int j = 0; j < BWD_AHEAD; ++j)
                if (!zero && v0 + j * BWD_THREADS < to) r[j] = load_16(xv + (int64_t)(v0 + j * BWD_THREADS) * VEC);
#pragma unroll
            for (int j = 0; j < BWD_AHEAD; ++j) {
                const int v = v0 + j * BWD_THREADS;
                if (v >= to) break;
                float f[VEC];
                values<T>(r[j], f);
                const int off = at_target - cut.index(v);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    f[i] = of(f[i]);
                    if (off == i) f[i] += a;
                    if (zero) f[i] = 0.f;
                }
                if constexpr (sizeof(T) == 4)
                    *reinterpret_cast<float4 *>(gv + (int64_t)v * VEC) = make_float4(f[0], f[1], f[2], f[3]);
                else {
                    DsqRaw8<T> out;
                    dsq_pack8(f, out);
                    dsq_store8(gv + (int64_t)v * VEC, out);
                }
            }
        }
    }
}

// Blocks of a row: as many as leave each a turn's work and the SMs no more than one each (rows of 128000 bf16 with five
// alternatives: 40 rows 10.2 us with two, 13.6 with one, 11.5 with four; 74 rows 11.2 with two, 14.2 with one; 100 rows 14.9
// with two, 14.5 with one).
int cluster_of(int64_t M, int64_t V, int threads, int vec)
{
    const int sms = dsq_sm_count() > 0 ? dsq_sm_count() : 148;
    int c = 1;
    while (c < MAX_CLUSTER && M * c * 2 <= sms && V >= (int64_t)threads * vec * 2 * c) c *= 2;
    return c;
}

template <class T, int THREADS> int fwd_launch(FwdParams &p, int64_t M, cudaStream_t s)
{
    const auto kernel = p.top > 0 ? logprob_fwd_kernel<T, true, THREADS> : logprob_fwd_kernel<T, false, THREADS>;
    return dsq_launch(kernel, dim3((unsigned)(M * p.cluster)), dim3(THREADS), 0, s, dsq_launch_hooks().pdl, p.cluster, p);
}

// Small blocks where there are rows enough to fill the SMs with them: some are between their passes while others read
// (the same rows: 148 of them 14.9 us with 512 threads, 18.8 with 256; 300 rows 30.9 and 32.2; 500 rows 39.5 and 36.2; 1024
// rows 65.2 and 58.3; 4096 rows 232 and 198).
template <class T> int fwd_pick(FwdParams &p, int64_t M, cudaStream_t s)
{
    const int sms = dsq_sm_count() > 0 ? dsq_sm_count() : 148;
    p.cluster = cluster_of(M, p.V, 512, vec_of<T>());
    return M >= 2 * sms ? fwd_launch<T, 256>(p, M, s) : fwd_launch<T, 512>(p, M, s);
}

template <class T> int bwd_launch(BwdParams &p, int64_t M, cudaStream_t s)
{
    const uintptr_t x = (uintptr_t)p.x, g = (uintptr_t)p.grad;
    const bool same = (x & 15) == (g & 15) && (p.ld - p.grad_ld) % vec_of<T>() == 0;
    p.segments = (p.V + bwd_segment<T>() - 1) / bwd_segment<T>();
    if (M * p.segments > 0x7FFFFFFF) return DSQ_ERR_SIZE;
    const dim3 grid((unsigned)(M * p.segments));
    const int pdl = dsq_launch_hooks().pdl;
    return same ? dsq_launch(logprob_bwd_kernel<T, true>, grid, dim3(BWD_THREADS), 0, s, pdl, 0, p)
                : dsq_launch(logprob_bwd_kernel<T, false>, grid, dim3(BWD_THREADS), 0, s, pdl, 0, p);
}

bool aligned_to(const void *p, int size) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(size - 1)) == 0; }

int check_rows(int64_t M, int64_t V, int64_t ld, int dtype, float scale)
{
    if (!dsq_is_float_type(dtype)) return DSQ_ERR_UNSUPPORTED;
    if (M <= 0 || V <= 0 || ld < V) return DSQ_ERR_SHAPE;
    if (V > 1 << 30 || M > 1 << 28) return DSQ_ERR_SIZE;
    if (!(scale > 0.f && scale <= MAX_SCALE)) return DSQ_ERR_RANGE;
    return DSQ_OK;
}

}  // namespace

extern "C" {

int dsq_logprob_fwd(const void *logits, int64_t ld, int64_t M, int64_t V, int dtype, const int64_t *targets,
                    float scale, int top, float *logp, float *entropy, float *lse, int64_t *top_ids,
                    float *top_logp, void *stream)
{
    if (!logits || (!logp && !entropy && !lse && !top_ids && !top_logp) || (logp && !targets)) return DSQ_ERR_NULL;
    const int st = check_rows(M, V, ld, dtype, scale);
    if (st) return st;
    if (top < 0 || top > V || (top == 0) != (!top_ids && !top_logp)) return DSQ_ERR_SHAPE;
    if (top > MAX_TOP) return DSQ_ERR_UNSUPPORTED;
    if (!aligned_to(logits, dtype == DSQ_F32 ? 4 : 2) || !aligned_to(targets, 8) || !aligned_to(top_ids, 8) ||
        !aligned_to(logp, 4) || !aligned_to(entropy, 4) || !aligned_to(lse, 4) || !aligned_to(top_logp, 4))
        return DSQ_ERR_ALIGN;
    FwdParams p;
    p.x = logits; p.targets = targets;
    p.logp = logp; p.entropy = entropy; p.lse = lse; p.top_logp = top_logp; p.top_ids = top_ids;
    p.ld = ld;
    p.V = (int)V; p.top = top; p.cluster = 1;
    p.scale = scale;
    cudaStream_t s = (cudaStream_t)stream;
    switch (dtype) {
    case DSQ_F32: return fwd_pick<float>(p, M, s);
    case DSQ_BF16: return fwd_pick<__nv_bfloat16>(p, M, s);
    default: return fwd_pick<__half>(p, M, s);
    }
}

int dsq_logprob_bwd(const void *logits, int64_t ld, int64_t M, int64_t V, int dtype, const int64_t *targets,
                    float scale, const float *lse, const float *entropy, const float *grad_logp,
                    const float *grad_entropy, void *grad_logits, int64_t grad_ld, void *stream)
{
    if (!logits || !lse || !grad_logits || (!grad_logp && !grad_entropy) || (grad_logp && !targets) ||
        (grad_entropy && !entropy))
        return DSQ_ERR_NULL;
    const int st = check_rows(M, V, ld, dtype, scale);
    if (st) return st;
    if (grad_ld < V) return DSQ_ERR_SHAPE;
    const int size = dtype == DSQ_F32 ? 4 : 2;
    if (!aligned_to(logits, size) || !aligned_to(grad_logits, size) || !aligned_to(targets, 8) || !aligned_to(lse, 4) ||
        !aligned_to(entropy, 4) || !aligned_to(grad_logp, 4) || !aligned_to(grad_entropy, 4))
        return DSQ_ERR_ALIGN;
    BwdParams p;
    p.x = logits; p.targets = targets;
    p.lse = lse; p.entropy = entropy; p.g_logp = grad_logp; p.g_entropy = grad_entropy;
    p.grad = grad_logits;
    p.ld = ld; p.grad_ld = grad_ld;
    p.V = (int)V; p.segments = 1;
    p.scale = scale;
    cudaStream_t s = (cudaStream_t)stream;
    switch (dtype) {
    case DSQ_F32: return bwd_launch<float>(p, M, s);
    case DSQ_BF16: return bwd_launch<__nv_bfloat16>(p, M, s);
    default: return bwd_launch<__half>(p, M, s);
    }
}

}  // extern "C"
