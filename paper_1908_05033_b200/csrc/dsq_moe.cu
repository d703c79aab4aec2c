// A layer of experts for few tokens: the router's choice, and the chosen experts' gated layers on
// 4-bit weights with group scales (what stands in a decoder where dsq_wgemm_group would be twice).
//
//   mid = act(x W_gate^T) * (x W_up^T),   y_t = residual_t + sum_s weight_ts mid_ts W_out^T
//
// Two kernels behind one another, both bound by the bytes of the experts that anything goes to:
//   * A slot is a token's s-th choice.  Every block sorts the slots by expert (stable, in shared memory) and cuts
//     each expert's into groups of up to ROWS, the rows of a tensor-core tile.
//   * moe_in_kernel: a block has 16 columns of a group's gate and the same 16 of its other half; its
//     warps split K in chunks of 128 codes, each through a ring of stages of its own (cp.async, no
//     barrier between warps); their sums are added in a fixed order, and the activation makes mid
//     of them.
//   * moe_out_kernel: a block (or a cluster, where there are few columns) has 32 columns of all tokens; the
//     chunks of all groups, one behind the other, are cut evenly among the warps, so that every
//     block has the same work however the tokens are spread.  A warp adds a group's sums, times the tokens'
//     weights, to rows of its own in shared memory; at the end the warps' and the cluster's are added in a fixed
//     order: no atomics, no partial results in memory, no third launch.  Its first weights are on their
//     way while the kernel ahead still runs.
//   * Codes become bf16 or fp16 pairs in registers as in dsq_wgemm_group.cu; products are exact and
//     added in binary32.  mid goes as two bf16 numbers, hi + lo (16 bits of mantissa: bf16 alone would
//     add as much again to the error as rounding y does), as the upper and lower eight rows of a tile,
//     which for eight slots costs the tensor core nothing.
//   * Rows of x and mid come from L2 straight into the operands' registers, a chunk ahead.
#include "dsq_groups.h"
#include "dsq_ptx.cuh"
#include "dsq_tc_host.h"
#include "dsq_types.cuh"
#include "dsq_wgemm_group.cuh"

using namespace dsq_ptx;

namespace {

constexpr int WARPS = 8, THREADS = WARPS * 32, PASS_TOKENS = 64, MAX_TOP = 32, MAX_EXPERTS = 1024;
constexpr int MAX_SLOTS = PASS_TOKENS * MAX_TOP;

// ---- the router's choice ---------------------------------------------------------------
// A warp a token: the largest key among those below the last, k times.  ITEMS logits a lane in
// registers, or (0) read again every time.
struct RouteParams {
    const float *logits;
    int32_t *ids;
    float *weights;
    int64_t T;
    int E, k, renormalise;
};

// ordered as the values are (-0 as 0), NaN below all
__device__ __forceinline__ uint32_t order_of(float v)
{
    const uint32_t u = __float_as_uint(v + 0.f);
    return v != v ? 0u : (int)u < 0 ? ~u : u | 0x80000000u;
}

template <int ITEMS> __global__ void __launch_bounds__(128) route_kernel(const RouteParams p)
{
    const int lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    grid_dependency_wait();
    grid_launch_dependents();
    if (t >= p.T) return;
    const float *row = p.logits + t * p.E;
    float v[ITEMS ? ITEMS : 1];
    if (ITEMS) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) v[i] = lane + 32 * i < p.E ? row[lane + 32 * i] : 0.f;
    }
    // (order, index) of the last: everything is below it at first
    uint32_t last = ~0u;
    int last_at = -1;
    float mine = 0.f, first = 0.f;
    int my_id = 0;
    for (int s = 0; s < p.k; ++s) {
        uint32_t best = 0u;
        int at = p.E;
        auto take = [&](float x, int e) {
            const uint32_t o = order_of(x);
            if ((o < last || (o == last && e > last_at)) && (at == p.E || o > best)) {
                best = o;
                at = e;
            }
        };
        if (ITEMS) {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
                if (lane + 32 * i < p.E) take(v[i], lane + 32 * i);
        } else {
            for (int e = lane; e < p.E; e += 32) take(row[e], e);
        }
        last = __reduce_max_sync(~0u, best);
        last_at = (int)__reduce_min_sync(~0u, best == last ? (uint32_t)at : (uint32_t)p.E);
        const float value = row[last_at];
        if (s == 0) first = value;
        if (lane == s) {
            mine = value;
            my_id = last_at;
        }
    }
    // (of a row of nothing but -infinity: 0)
    const bool none = first == __uint_as_float(0xFF800000u);
    float e = lane < p.k ? expf(mine - first) : 0.f, sum = e;
    if (!p.renormalise) {
        sum = 0.f;
        for (int i = lane; i < p.E; i += 32) sum += expf(row[i] - first);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    if (lane < p.k) {
        p.ids[t * p.k + lane] = my_id;
        p.weights[t * p.k + lane] = none ? 0.f : e / sum;
    }
}

// ---- slots by expert ---------------------------------------------------------------------
struct Group {
    int expert, first, n;             // slots first .. first + n - 1 of the sorted ones
};
struct Slots {
    uint16_t sorted[MAX_SLOTS];
    uint32_t packed[MAX_SLOTS];       // groups: expert | first << 10 | (n - 1) << 22
    int start[MAX_EXPERTS];           // (counts, then where the next slot of an expert goes)
    int groups;
    __device__ __forceinline__ Group group(int i) const
    {
        const uint32_t v = packed[i];
        return {(int)(v & 1023), (int)(v >> 10 & 4095), (int)(v >> 22) + 1};
    }
};

// Sorts the slots whose expert there is; groups of up to `rows`.  All threads; ends with a barrier.
__device__ __forceinline__ void sort_slots(Slots &s, const int32_t *ids, int n, int E, int rows)
{
    const int lane = threadIdx.x & 31;
    for (int e = threadIdx.x; e < E; e += THREADS) s.start[e] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += THREADS) {
        const int id = ids[i];
        if (id >= 0 && id < E) atomicAdd(&s.start[id], 1);
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        int slots = 0, groups = 0;    // so far
        for (int e0 = 0; e0 < E; e0 += 32) {
            const int e = e0 + lane, count = e < E ? s.start[e] : 0, parts = (count + rows - 1) / rows;
            int a = count, b = parts;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int u = __shfl_up_sync(~0u, a, o), v = __shfl_up_sync(~0u, b, o);
                if (lane >= o) {
                    a += u;
                    b += v;
                }
            }
            const int first = slots + a - count, g = groups + b - parts;
            if (e < E) s.start[e] = first;
            for (int i = 0; i < parts; ++i)
                s.packed[g + i] = (uint32_t)e | (uint32_t)(first + i * rows) << 10 | (uint32_t)(min(rows, count - i * rows) - 1) << 22;
            slots += __shfl_sync(~0u, a, 31);
            groups += __shfl_sync(~0u, b, 31);
        }
        if (lane == 0) s.groups = groups;
        __syncwarp();
        for (int i0 = 0; i0 < n; i0 += 32) {
            int id = i0 + lane < n ? ids[i0 + lane] : -1;
            if (id < 0 || id >= E) id = -1;
            const uint32_t same = __match_any_sync(~0u, id);
            int at = id >= 0 ? s.start[id] : 0;
            __syncwarp();
            if (id >= 0) {
                s.sorted[at + __popc(same & ((1u << lane) - 1))] = (uint16_t)(i0 + lane);
                if (lane == 31 - __clz(same)) s.start[id] = at + __popc(same);
            }
            __syncwarp();
        }
    }
    __syncthreads();
}

// ---- products ------------------------------------------------------------------------------
struct MoeParams {
    const uint8_t *X, *W_in, *W_out;
    const float *s_in, *s_out, *weights;
    const int32_t *ids;
    uint16_t *mid;                    // hi rows of all slots, then lo rows, of pitch_mid bf16 each
    const void *residual;
    void *Y;
    int T, H, I, E, k, slots;
    int pitch_in, pitch_out, pitch_mid;      // bytes of a row of codes; elements
    int groups_in, groups_out;               // scales of a row
    uint32_t units_in, units_in_inv, units_out, units_out_inv;
    int odd, act, y_type;
};

// group of scales of a unit (dsq_wgemm_group.cuh)
__device__ __forceinline__ int scale_of(uint32_t unit, uint32_t units, uint32_t inv)
{
    return units == 1 ? (int)unit : (int)__umulhi(unit, inv);
}

template <int XT> __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if (XT == DSQ_BF16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
            "{%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
            "{%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void cp_async_4(uint32_t dst, const void *src, uint32_t src_bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(src_bytes) : "memory");
}
__device__ __forceinline__ uint4 load_16(const void *p)
{
    uint4 r;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}

// Codes of 8 NT columns and the scales of a chunk's 4 / GP units, as dsq_wgemm_group.cu keeps them.
template <int NT, int GP> struct Stage {
    static constexpr int W_BYTES = NT * 512, S_BYTES = (4 / GP) * NT * 32, BYTES = W_BYTES + S_BYTES;
};

// Copies of a chunk: column c of the stage is row(c) of the matrix of codes (negative: none).
template <int NT, int GP, class Row>
__device__ __forceinline__ void copy_chunk(uint32_t at, const uint8_t *W, int pitch, const float *scales, int64_t rows, int groups,
                                           uint32_t units, uint32_t inv, int chunk, Row row)
{
    const int lane = threadIdx.x & 31, n = lane >> 2, j = lane & 3;
    const int k_at = chunk * 64 + 16 * j;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int64_t r = row(8 * t + n);
        const bool in = r >= 0 && k_at < pitch;
        cp_async_16(at + t * 512 + n * 64 + ((j ^ (n >> 1)) & 3) * 16, in ? W + r * pitch + k_at : W, in ? 16u : 0u);
    }
#pragma unroll
    for (int s = lane; s < (4 / GP) * NT * 8; s += 32) {
        const int g = scale_of((uint32_t)(chunk * (4 / GP) + s / (8 * NT)), units, inv);
        const int64_t r = row(s % (8 * NT));
        const bool in = r >= 0 && g < groups;
        cp_async_4(at + Stage<NT, GP>::W_BYTES + s * 4, in ? scales + (int64_t)g * rows + r : scales, in ? 4u : 0u);
    }
}

// A lane's rows of a tile's operand: 16 bytes of each of a chunk's four pieces, of rows n and n + 8 of each tile.
template <int TILES> struct Rows { uint4 x[TILES][2][4]; };

// Sums of a chunk: total += scale (sum of x v).  `refill(tile, half, piece)`: what is loaded where a piece was.
template <int XT, int TILES, int NT, int GP, class Refill>
__device__ __forceinline__ void multiply(uint32_t at, uint32_t base, Rows<TILES> &r, float (&total)[TILES][NT][4], Refill refill)
{
    const int lane = threadIdx.x & 31, n = lane >> 2, j = lane & 3;
    const uint32_t as = at + Stage<NT, GP>::W_BYTES;
    float acc[TILES][NT][4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (q % GP == 0) {
#pragma unroll
            for (int m = 0; m < TILES; ++m)
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[m][t][e] = 0.f;
        }
        uint32_t a[TILES][2][4];
#pragma unroll
        for (int m = 0; m < TILES; ++m) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint4 v = r.x[m][h][q];
                // elements (2 s, 2 s + 4) and (2 s + 1, 2 s + 5), as the codes come out of their words
                a[m][0][h] = __byte_perm(v.x, v.z, 0x5410);
                a[m][0][h + 2] = __byte_perm(v.x, v.z, 0x7632);
                a[m][1][h] = __byte_perm(v.y, v.w, 0x5410);
                a[m][1][h + 2] = __byte_perm(v.y, v.w, 0x7632);
                refill(m, h, q);
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint32_t w = lds_32(at + t * 512 + n * 64 + ((q ^ (n >> 1)) & 3) * 16 + 4 * j);
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const uint32_t b0 = dsq_value_pair<XT>(w, 2 * s, base), b1 = dsq_value_pair<XT>(w, 2 * s + 1, base);
#pragma unroll
                for (int m = 0; m < TILES; ++m) mma<XT>(acc[m][t], a[m][s], b0, b1);
            }
        }
        if (q % GP == GP - 1) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const uint2 sv = lds_64(as + (q / GP * NT * 8 + 8 * t + 2 * j) * 4);
                const float s0 = __uint_as_float(sv.x), s1 = __uint_as_float(sv.y);
#pragma unroll
                for (int m = 0; m < TILES; ++m) {
                    total[m][t][0] = __fmaf_rn(acc[m][t][0], s0, total[m][t][0]);
                    total[m][t][1] = __fmaf_rn(acc[m][t][1], s1, total[m][t][1]);
                    total[m][t][2] = __fmaf_rn(acc[m][t][2], s0, total[m][t][2]);
                    total[m][t][3] = __fmaf_rn(acc[m][t][3], s1, total[m][t][3]);
                }
            }
        }
    }
}

__device__ __forceinline__ float activated(float g, int act)
{
    if (act == DSQ_SILU) return g / (1.f + expf(-g));
    const float u = 0.7978845608028654f * __fmaf_rn(0.044715f * g * g, g, g);
    return 0.5f * g * (1.f + tanhf(u));
}

// HALF: groups of up to 8 slots (the lower half of a tile), else 16
template <int XT, bool HALF, int GP, int STAGES>
__global__ void __launch_bounds__(THREADS, 2) moe_in_kernel(const __grid_constant__ MoeParams p)
{
    constexpr int NT = 4, ROWS = HALF ? 8 : 16, COLS = 16;
    using S = Stage<NT, GP>;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ Slots slots;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = lane >> 2, j = lane & 3;
    const int c0 = blockIdx.x * COLS;
    const int chunks = (p.H + 127) >> 7, turns = warp < chunks ? (chunks - warp - 1) / WARPS + 1 : 0;
    const uint32_t ring = smem_u32(smem) + (uint32_t)(warp * STAGES * S::BYTES), base = dsq_value_base<XT>(p.odd);
    grid_dependency_wait();
    grid_launch_dependents();
    sort_slots(slots, p.ids, p.slots, p.E, ROWS);
    for (int gi = blockIdx.y; gi < slots.groups; gi += gridDim.y) {
        const Group g = slots.group(gi);
        const int64_t row0 = (int64_t)g.expert * 2 * p.I + c0;
        auto row = [&](int c) { return c0 + (c & 15) < p.I ? row0 + (c & 15) + (c < 16 ? 0 : p.I) : (int64_t)-1; };
        auto issue = [&](int i) {
            if (i < turns)
                copy_chunk<NT, GP>(ring + (uint32_t)(i % STAGES * S::BYTES), p.W_in, p.pitch_in, p.s_in, (int64_t)p.E * 2 * p.I,
                                   p.groups_in, p.units_in, p.units_in_inv, warp + i * WARPS, row);
            cp_async_commit();
        };
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s) issue(s);
        const uint8_t *x[2];
        bool has[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            has[h] = n + 8 * h < g.n;
            x[h] = p.X + (has[h] ? (int64_t)(slots.sorted[g.first + n + 8 * h] / p.k) * p.H * 2 : 0) + 16 * j;
        }
        Rows<1> r;
        auto load = [&](int i, int h, int q) {
            const int at = (warp + i * WARPS) * 256 + 64 * q;
            r.x[0][h][q] = has[h] && i < turns && at + 16 * j < 2 * p.H ? load_16(x[h] + at) : make_uint4(0u, 0u, 0u, 0u);
        };
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int q = 0; q < 4; ++q) load(0, h, q);
        float total[1][NT][4] = {};
#pragma unroll 1
        for (int i = 0; i < turns; ++i) {
            cp_async_wait<STAGES - 2>();
            __syncwarp();             // every lane's copies of this stage are here, and the last stage has been read
            issue(i + STAGES - 1);
            multiply<XT, 1, NT, GP>(ring + (uint32_t)(i % STAGES * S::BYTES), base, r, total,
                                    [&](int, int h, int q) { load(i + 1, h, q); });
        }
        // the warps' sums, added in a fixed order
        cp_async_wait<0>();
        __syncthreads();
        float4 *part = reinterpret_cast<float4 *>(smem);        // [WARPS][NT][32]
#pragma unroll
        for (int t = 0; t < NT; ++t)
            part[(warp * NT + t) * 32 + lane] = make_float4(total[0][t][0], total[0][t][1], total[0][t][2], total[0][t][3]);
        __syncthreads();
        const float unit = dsq_value_unit<XT>(p.odd);
        const float *sums = reinterpret_cast<const float *>(smem);
        for (int e = threadIdx.x; e < ROWS * COLS; e += THREADS) {
            const int rr = e / COLS, c = e % COLS;
            if (rr >= g.n) break;
            const int at = ((c >> 3) * 32 + (rr & 7) * 4 + ((c & 7) >> 1)) * 4 + 2 * (rr >> 3) + (c & 1);
            float gate = 0.f, up = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                gate += sums[w * NT * 128 + at];
                up += sums[w * NT * 128 + 2 * 128 + at];
            }
            // (columns behind the last are zeros up to the row's pitch)
            float v = c0 + c < p.I ? activated(gate * unit, p.act) * (up * unit) : 0.f;
            const __nv_bfloat16 hi = __float2bfloat16_rn(v);
            const float rest = v - __bfloat162float(hi);
            // (an infinity or a NaN has no rest)
            const __nv_bfloat16 lo = __float2bfloat16_rn(rest == rest ? rest : 0.f);
            const int64_t to = (int64_t)slots.sorted[g.first + rr] * p.pitch_mid + c0 + c;
            p.mid[to] = __bfloat16_as_ushort(hi);
            p.mid[to + (int64_t)p.slots * p.pitch_mid] = __bfloat16_as_ushort(lo);
        }
        __syncthreads();
    }
}

template <int TILES, int GP, int STAGES>
__global__ void __launch_bounds__(THREADS, TILES == 1 ? 2 : 1) moe_out_kernel(const __grid_constant__ MoeParams p, int cluster)
{
    constexpr int NT = 4, ROWS = 8 * TILES, COLS = 8 * NT;
    using S = Stage<NT, GP>;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ Slots slots;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = lane >> 2, j = lane & 3;
    const int rank = cluster > 1 ? (int)cluster_ctarank() : 0;
    const int64_t c0 = (int64_t)(blockIdx.x / cluster) * COLS;
    const int chunks = (p.I + 127) >> 7;
    const uint32_t ring = smem_u32(smem) + (uint32_t)(warp * STAGES * S::BYTES), base = dsq_value_base<DSQ_BF16>(p.odd);
    // [WARPS][T][COLS]; the warp's own
    float *sums = reinterpret_cast<float *>(smem + WARPS * STAGES * S::BYTES), *mine = sums + warp * p.T * COLS;
    // Ahead of the wait: ids, codes and scales are older than the kernel ahead (moe_in_kernel, which
    // waited for all that was in front of it before it let this one start).
    sort_slots(slots, p.ids, p.slots, p.E, ROWS);
    // this warp's share of the chunks of all groups
    const int64_t all = (int64_t)slots.groups * chunks, share = rank * WARPS + warp, shares = cluster * WARPS;
    const int q0 = (int)(all * share / shares), q1 = (int)(all * (share + 1) / shares);
    int ig = q0 / chunks, ic = q0 - ig * chunks;                // of the next copy
    auto issue = [&](int i) {
        if (i < q1) {
            const int64_t row0 = (int64_t)(slots.packed[ig] & 1023) * p.H + c0;
            copy_chunk<NT, GP>(ring + (uint32_t)((i - q0) % STAGES * S::BYTES), p.W_out, p.pitch_out, p.s_out, (int64_t)p.E * p.H,
                               p.groups_out, p.units_out, p.units_out_inv, ic,
                               [&](int c) { return c0 + c < p.H ? row0 + c : (int64_t)-1; });
            if (++ic == chunks) {
                ic = 0;
                ++ig;
            }
        }
        cp_async_commit();
    };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) issue(q0 + s);
    for (int i = lane; i < p.T * COLS; i += 32) mine[i] = 0.f;
    __syncwarp();
    grid_dependency_wait();
    grid_launch_dependents();

    // rows of the chunk that is loaded next
    int lg = q0 / chunks, lc = q0 - lg * chunks;
    const uint16_t *x[TILES];
    bool has[TILES];
    const int64_t lo = (int64_t)p.slots * p.pitch_mid;
    auto rows_of = [&]() {
        if (lg >= slots.groups) return;
        const Group g = slots.group(lg);
#pragma unroll
        for (int m = 0; m < TILES; ++m) {
            has[m] = n + 8 * m < g.n;
            x[m] = p.mid + (has[m] ? (int64_t)slots.sorted[g.first + n + 8 * m] * p.pitch_mid : 0) + 8 * j;
        }
    };
    Rows<TILES> r;
    auto load = [&](bool on, int m, int h, int q) {
        const int at = lc * 128 + 32 * q;
        r.x[m][h][q] = on && has[m] && at + 8 * j < p.pitch_mid ? load_16(x[m] + (h ? lo : 0) + at) : make_uint4(0u, 0u, 0u, 0u);
    };
    rows_of();
#pragma unroll
    for (int m = 0; m < TILES; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int q = 0; q < 4; ++q) load(q0 < q1, m, h, q);
    float total[TILES][NT][4] = {};
    int cg = lg, cc = lc;                                       // of the chunk at hand
#pragma unroll 1
    for (int i = q0; i < q1; ++i) {
        cp_async_wait<STAGES - 2>();
        __syncwarp();
        issue(i + STAGES - 1);
        if (++lc == chunks) {
            lc = 0;
            ++lg;
            rows_of();
        }
        multiply<DSQ_BF16, TILES, NT, GP>(ring + (uint32_t)((i - q0) % STAGES * S::BYTES), base, r, total,
                                          [&](int m, int h, int q) { load(i + 1 < q1, m, h, q); });
        if (++cc < chunks && i + 1 < q1) continue;
        // the group's sums to the tokens' rows, one slot after the other (two may be the same token's)
        const Group g = slots.group(cg);
#pragma unroll
        for (int m = 0; m < TILES; ++m)
            for (int rr = 0; rr < 8 && 8 * m + rr < g.n; ++rr) {
                if (n == rr) {
                    const int slot = slots.sorted[g.first + 8 * m + rr], token = slot / p.k;
                    const float w = p.weights[slot];
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        float2 *to = reinterpret_cast<float2 *>(mine + token * COLS + 8 * t + 2 * j);
                        float2 v = *to;
                        v.x = __fmaf_rn(total[m][t][0] + total[m][t][2], w, v.x);
                        v.y = __fmaf_rn(total[m][t][1] + total[m][t][3], w, v.y);
                        *to = v;
                    }
                }
                __syncwarp();
            }
#pragma unroll
        for (int m = 0; m < TILES; ++m)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) total[m][t][e] = 0.f;
        cc = 0;
        ++cg;
    }
    cp_async_wait<0>();
    __syncthreads();
    // the warps' rows, into the first one's place
    for (int e = threadIdx.x; e < p.T * COLS; e += THREADS) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) s += sums[w * p.T * COLS + e];
        sums[e] = s;
    }
    if (cluster > 1) cluster_sync_all();
    else __syncthreads();
    const float unit = dsq_value_unit<DSQ_BF16>(p.odd);
    for (int e = rank * THREADS + threadIdx.x; e < p.T * COLS; e += cluster * THREADS) {
        float s = 0.f;
        if (cluster == 1) s = sums[e];
        else
            for (int c = 0; c < cluster; ++c) s += __uint_as_float(ld_cluster_32(map_to_cta(smem_u32(sums + e), c)));
        const int64_t col = c0 + e % COLS;
        if (col >= p.H) continue;
        const int64_t to = (int64_t)(e / COLS) * p.H + col;
        s *= unit;
        if (p.y_type == DSQ_F32) {
            if (p.residual) s += ((const float *)p.residual)[to];
            ((float *)p.Y)[to] = s;
        } else if (p.y_type == DSQ_BF16) {
            if (p.residual) s += __bfloat162float(((const __nv_bfloat16 *)p.residual)[to]);
            ((__nv_bfloat16 *)p.Y)[to] = __float2bfloat16_rn(s);
        } else {
            if (p.residual) s += __half2float(((const __half *)p.residual)[to]);
            ((__half *)p.Y)[to] = __float2half_rn(s);
        }
    }
    if (cluster > 1) cluster_sync_all();      // nobody leaves while its sums are read
}

// ---- host ------------------------------------------------------------------------------------
constexpr int IN_STAGES = 4, OUT_STAGES = 3;

template <int XT, int GP> int launch_in(const MoeParams &p, cudaStream_t s)
{
    using S = Stage<4, GP>;
    constexpr int bytes = WARPS * IN_STAGES * S::BYTES;
    static_assert(bytes >= WARPS * 4 * 512 && bytes <= 100 * 1024, "shared memory");
    const dim3 grid((unsigned)((p.I + 15) / 16), (unsigned)(p.slots < p.E ? p.slots : p.E));
    const bool half = p.T <= 8;
    static std::atomic<unsigned long long> configured[2];
    const auto kernel = half ? moe_in_kernel<XT, true, GP, IN_STAGES> : moe_in_kernel<XT, false, GP, IN_STAGES>;
    const int st = dsq_allow_smem((const void *)kernel, bytes, &configured[half]);
    if (st) return st;
    return dsq_launch(kernel, grid, dim3(THREADS), (size_t)bytes, s, dsq_launch_hooks().pdl, 0, p);
}

template <int TILES, int GP> int launch_out(const MoeParams &p, cudaStream_t s)
{
    using S = Stage<4, GP>;
    constexpr int ring = WARPS * OUT_STAGES * S::BYTES, row = WARPS * 32 * 4, most = ring + PASS_TOKENS * row;
    static_assert(most <= 200 * 1024, "shared memory");
    static std::atomic<unsigned long long> configured;
    const auto kernel = moe_out_kernel<TILES, GP, OUT_STAGES>;
    const int st = dsq_allow_smem((const void *)kernel, most, &configured);
    if (st) return st;
    const int tiles = (p.H + 31) / 32, sms = dsq_sm_count() > 0 ? dsq_sm_count() : 148;
    int cluster = 1;
    while (cluster < 8 && tiles * cluster * 2 <= 2 * sms) cluster *= 2;
    return dsq_launch(kernel, dim3((unsigned)(tiles * cluster)), dim3(THREADS), (size_t)(ring + p.T * row), s,
                      dsq_launch_hooks().pdl, cluster, p, cluster);
}

template <int GP_IN> int pick_in(const MoeParams &p, int x_type, cudaStream_t s)
{
    return x_type == DSQ_BF16 ? launch_in<DSQ_BF16, GP_IN>(p, s) : launch_in<DSQ_F16, GP_IN>(p, s);
}
template <int GP> int pick_out(const MoeParams &p, cudaStream_t s)
{
    return p.T <= 8 ? launch_out<1, GP>(p, s) : launch_out<2, GP>(p, s);
}

int pitch_of_mid(int64_t I) { return (int)((I + 15) / 16 * 16); }

// a group longer than the row is the row
int64_t group_of_row(int64_t K, int64_t group) { return dsq_group_count(K, group) == 1 ? (K + 127) / 128 * 128 : group; }

void set_units(int64_t group, int gp, uint32_t *units, uint32_t *inv)
{
    DsqGroupGemm g;
    g.set_units(group, gp);
    *units = g.units;
    *inv = g.units_inv;
}

}  // namespace

extern "C" {

int dsq_moe_route(const float *logits, int64_t T, int64_t E, int k, int renormalise, int32_t *ids, float *weights,
                  void *stream)
{
    if (!logits || !ids || !weights) return DSQ_ERR_NULL;
    if (T <= 0 || E <= 0 || k <= 0 || k > E) return DSQ_ERR_SHAPE;
    if (T > 1 << 28 || E > 1 << 20 || k > MAX_TOP) return DSQ_ERR_SIZE;
    if (!dsq_aligned16(logits) || !dsq_aligned16(ids) || !dsq_aligned16(weights)) return DSQ_ERR_ALIGN;
    const RouteParams p = {logits, ids, weights, T, (int)E, k, renormalise != 0};
    const auto kernel = E <= 64 ? route_kernel<2> : E <= 256 ? route_kernel<8> : route_kernel<0>;
    return dsq_launch(kernel, dim3((unsigned)((T + 3) / 4)), dim3(128), 0, (cudaStream_t)stream, dsq_launch_hooks().pdl, 0, p);
}

size_t dsq_moe_workspace_bytes(int64_t T, int64_t I, int k)
{
    if (T <= 0 || I <= 0 || I > 1 << 24 || k <= 0 || k > MAX_TOP) return DSQ_WS_BYTES;
    return DSQ_WS_BYTES + (size_t)(T < PASS_TOKENS ? T : PASS_TOKENS) * (size_t)k * (size_t)pitch_of_mid(I) * 4;
}

int dsq_moe_group(const void *X, int x_type, const int32_t *ids, const float *weights, const void *W_in,
                  const float *scales_in, const void *W_out, const float *scales_out, int64_t T, int64_t H, int64_t I,
                  int64_t E, int k, int bits, int64_t group, float w_offset, int activation, const void *residual,
                  int y_type, void *Y, void *workspace, size_t ws_bytes, void *stream)
{
    if (!X || !ids || !weights || !W_in || !scales_in || !W_out || !scales_out || !Y || !workspace) return DSQ_ERR_NULL;
    if (T <= 0 || H <= 0 || I <= 0 || E <= 0 || k <= 0) return DSQ_ERR_SHAPE;
    if (T > 1 << 20 || H > DSQ_GROUPS_MAX_K || I > DSQ_GROUPS_MAX_K || E > MAX_EXPERTS || k > MAX_TOP) return DSQ_ERR_SIZE;
    int st = dsq_check_groups(E * 2 * I, H, bits, group);
    if (!st) st = dsq_check_groups(E * H, I, bits, group);
    if (st) return st;
    if (!dsq_finite(w_offset)) return DSQ_ERR_RANGE;
    if ((x_type != DSQ_BF16 && x_type != DSQ_F16) || !dsq_is_float_type(y_type) || (w_offset != 0.0f && w_offset != 0.5f) ||
        (activation != DSQ_SILU && activation != DSQ_GELU_TANH))
        return DSQ_ERR_UNSUPPORTED;
    const void *aligned[] = {X, ids, weights, W_in, scales_in, W_out, scales_out, residual, Y, workspace};
    for (const void *a : aligned)
        if (!dsq_aligned16(a)) return DSQ_ERR_ALIGN;
    if (H % 8 != 0) return DSQ_ERR_ALIGN;
    if (ws_bytes < dsq_moe_workspace_bytes(T, I, k)) return DSQ_ERR_SIZE;
    const int64_t g_in = group_of_row(H, group), g_out = group_of_row(I, group);
    const int gp_in = dsq_group_pieces(g_in), gp_out = dsq_group_pieces(g_out);
    MoeParams p;
    p.W_in = (const uint8_t *)W_in; p.W_out = (const uint8_t *)W_out;
    p.s_in = scales_in; p.s_out = scales_out;
    p.mid = (uint16_t *)((char *)workspace + DSQ_WS_BYTES);
    p.H = (int)H; p.I = (int)I; p.E = (int)E; p.k = k;
    p.pitch_in = (int)dsq_row_pitch(H, 4); p.pitch_out = (int)dsq_row_pitch(I, 4); p.pitch_mid = pitch_of_mid(I);
    p.groups_in = (int)dsq_group_count(H, g_in); p.groups_out = (int)dsq_group_count(I, g_out);
    set_units(g_in, gp_in, &p.units_in, &p.units_in_inv);
    set_units(g_out, gp_out, &p.units_out, &p.units_out_inv);
    p.odd = w_offset == 0.5f; p.act = activation; p.y_type = y_type;
    cudaStream_t s = (cudaStream_t)stream;
    const int64_t y_size = y_type == DSQ_F32 ? 4 : 2;
    for (int64_t t = 0; t < T; t += PASS_TOKENS) {
        p.T = (int)(T - t < PASS_TOKENS ? T - t : PASS_TOKENS);
        p.slots = p.T * k;
        p.X = (const uint8_t *)X + t * H * 2;
        p.ids = ids + t * k; p.weights = weights + t * k;
        p.residual = residual ? (const char *)residual + t * H * y_size : nullptr;
        p.Y = (char *)Y + t * H * y_size;
        st = gp_in == 4 ? pick_in<4>(p, x_type, s) : gp_in == 2 ? pick_in<2>(p, x_type, s) : pick_in<1>(p, x_type, s);
        if (!st) st = gp_out == 4 ? pick_out<4>(p, s) : gp_out == 2 ? pick_out<2>(p, s) : pick_out<1>(p, s);
        if (st) return st;
    }
    return DSQ_OK;
}

}  // extern "C"
