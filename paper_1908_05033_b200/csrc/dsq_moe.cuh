// What the kernels for layers of experts share (dsq_moe.cu: groups of up to four slots, on digits of 8 bits;
// dsq_moe_wide.cu: of up to sixteen, on 16 bits).
#pragma once

#include "dsq_groups.h"
#include "dsq_pairs.cuh"
#include "dsq_ptx.cuh"
#include "dsq_tc_host.h"
#include "dsq_types.cuh"
#include "dsq_wgemm_group.cuh"

namespace dsq_moe {

using namespace dsq_ptx;

constexpr int PASS_TOKENS = 64, MAX_TOP = 32, MAX_EXPERTS = 1024;      // tokens of a pass over the weights

// ---- slots by expert
// a group as the kernels read it, in one access
struct alignas(64) Group {
    int expert, n, unused[2];
    uint16_t slot[16];
};
// what lies in the workspace
struct Work {
    int *groups;                      // how many
    Group *group;                     // by expert, the slots of an expert in their order
    // digits: [T][chunks_in], [slots][chunks_out], what the highest digit stands for; 16 bits: [T], [slots], what 1 stands for
    float *x_step, *mid_step;
    // digits: [T][chunks_in][512], [slots][chunks_out][512]; 16 bits: [T][chunks_in][256], [slots][chunks_out][512]
    uint8_t *x, *mid_rows;
    float *mid;                       // [slots][128 chunks_out]
    float *part;                      // 16 bits: [slots][H], what a slot adds to its token (where mid was)
};
struct MoeParams {
    Work w;
    const uint8_t *X, *W_in, *W_out;
    const float *s_in, *s_out, *weights;
    const int32_t *ids;
    const void *residual;
    void *Y;
    int T, H, I, E, k, slots;
    int pitch_in, pitch_out;                 // bytes of a row of codes
    int chunks_in, chunks_out;               // of 128 codes in a row
    int groups_in, groups_out;               // scales of a row
    uint32_t units_in, units_in_inv, units_out, units_out_inv;
    int odd, act, y_type;
    int rows;                                // slots of a group: 4 (digits), 8 or 16 (16 bits)
    int scaled;                              // 16 bits: x, in bf16, as fp16 times a power of two
    // No call has more groups: blocks are launched for so many (as many as experts, each taking several groups in turn where
    // all tokens go to few experts: 64 tokens, one expert of 2048 to 768, 69 us, with all at once 23; three of 11, 75 and 55).
    int groups_most() const { const int most = E + slots / rows; return slots < most ? slots : most; }
};
__device__ __forceinline__ uint4 load_16(const void *p)
{
    uint4 r;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}

// Up to 32 slots, one a lane of a warp: groups in the order of their first slots, unless an expert has more than one.
struct Few {
    int id;                           // of the lane's slot, -1: none
    uint32_t same, firsts;            // lanes of this lane's expert; the first lane of each expert
    bool fit;                         // no expert has more than one group
    __device__ __forceinline__ explicit Few(const MoeParams &p)
    {
        const int lane = threadIdx.x & 31;
        id = lane < p.slots ? p.ids[lane] : -1;
        if (id < 0 || id >= p.E) id = -1;
        same = __match_any_sync(~0u, id);
        firsts = __ballot_sync(~0u, id >= 0 && (same & below()) == 0u);
        fit = !__any_sync(~0u, id >= 0 && __popc(same) > p.rows);
    }
    __device__ __forceinline__ static uint32_t below() { return (1u << (threadIdx.x & 31)) - 1; }
    __device__ __forceinline__ int groups() const { return __popc(firsts); }
    // group i (there is one): its expert, its slots as bits
    __device__ __forceinline__ void group(int i, int &expert, uint32_t &slots) const
    {
        const uint32_t of = __ballot_sync(~0u, (firsts >> (threadIdx.x & 31) & 1) && __popc(firsts & below()) == i);
        expert = __shfl_sync(~0u, id, __ffs(of) - 1);
        slots = __shfl_sync(~0u, same, __ffs(of) - 1);
    }
};

// Sorts the slots whose expert there is, and cuts them into groups.  A block.
struct Sorting { int count[MAX_EXPERTS], group[MAX_EXPERTS]; };
__device__ __forceinline__ void sort_slots(const MoeParams &p, Sorting &s)
{
    const int lane = threadIdx.x & 31, E = p.E, n = p.slots, rows = p.rows, shift = rows == 16 ? 4 : rows == 8 ? 3 : 2;
    if (n <= 32) {
        if (threadIdx.x < 32) {
            const Few few(p);
            if (few.fit) {
                const int before = __popc(few.same & Few::below());
                if (few.id >= 0) {
                    Group *g = p.w.group + __popc(few.firsts & ((1u << (__ffs(few.same) - 1)) - 1));
                    g->slot[before] = (uint16_t)lane;
                    if (before == 0) {
                        g->expert = few.id;
                        g->n = __popc(few.same);
                    }
                }
                if (lane == 0) *p.w.groups = few.groups();
            }
            if (lane == 0) s.group[0] = few.fit ? -1 : 0;
        }
        __syncthreads();
        if (s.group[0] < 0) return;
    }
    for (int e = threadIdx.x; e < E; e += blockDim.x) s.count[e] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const int id = p.ids[i];
        if (id >= 0 && id < E) atomicAdd(&s.count[id], 1);
    }
    __syncthreads();
    if (threadIdx.x >= 32) return;
    int groups = 0;                   // so far
    for (int e0 = 0; e0 < E; e0 += 32) {
        const int e = e0 + lane, count = e < E ? s.count[e] : 0, parts = (count + rows - 1) >> shift;
        int b = parts;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(~0u, b, o);
            if (lane >= o) b += v;
        }
        const int g = groups + b - parts;
        if (e < E) {
            s.count[e] = 0;
            s.group[e] = g;
        }
        for (int i = 0; i < parts; ++i) {
            p.w.group[g + i].expert = e;
            p.w.group[g + i].n = min(rows, count - i * rows);
        }
        groups += __shfl_sync(~0u, b, 31);
    }
    if (lane == 0) *p.w.groups = groups;
    __syncwarp();
    for (int i0 = 0; i0 < n; i0 += 32) {
        int id = i0 + lane < n ? p.ids[i0 + lane] : -1;
        if (id < 0 || id >= E) id = -1;
        const uint32_t same = __match_any_sync(~0u, id);
        const int at = id >= 0 ? s.count[id] : 0;
        __syncwarp();
        if (id >= 0) {
            const int pos = at + __popc(same & ((1u << lane) - 1));
            p.w.group[s.group[id] + (pos >> shift)].slot[pos & (rows - 1)] = (uint16_t)(i0 + lane);
            if (lane == 31 - __clz(same)) s.count[id] = at + __popc(same);
        }
        __syncwarp();
    }
}

constexpr int NT = 4;                 // tiles of eight columns that a warp has

// ---- products ------------------------------------------------------------------------------
// group of scales of a unit (dsq_wgemm_group.cuh)
__device__ __forceinline__ int scale_of(uint32_t unit, uint32_t units, uint32_t inv)
{
    return units == 1 ? (int)unit : (int)__umulhi(unit, inv);
}

__device__ __forceinline__ void cp_async_4(uint32_t dst, const void *src, uint32_t src_bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(src_bytes) : "memory");
}

// Codes of 8 NT columns and the scales of a chunk's 4 / GP units, as dsq_wgemm_group.cu keeps them.
template <int NT, int GP> struct Stage {
    static constexpr int W_BYTES = NT * 512, S_BYTES = (4 / GP) * NT * 32, BYTES = W_BYTES + S_BYTES;
};

// A warp's copies of codes and scales, every `by`-th chunk from `first` on, to the places of a ring of STAGES in turn.
// (Columns behind the last are the last: their sums are not used.  A copy of 0 bytes reads nothing, wherever it points.)
template <int NT, int GP, int STAGES> struct Copies {
    const uint8_t *w[NT];             // 16-byte piece j of this lane's columns, of the next chunk
    const float *scale;               // of the column whose scales this lane copies
    uint32_t to, to_first, to_scale;  // places in shared memory; the scales' behind the codes'
    int chunk, by;
    __device__ __forceinline__ void start(uint32_t ring, int first, int by_)
    {
        const int lane = threadIdx.x & 31, n = lane >> 2, j = lane & 3;
        to = to_first = ring + n * 64 + ((j ^ (n >> 1)) & 3) * 16;
        to_scale = Stage<NT, GP>::W_BYTES + lane * 4 - (n * 64 + ((j ^ (n >> 1)) & 3) * 16);
        chunk = first;
        by = by_;
#pragma unroll
        for (int t = 0; t < NT; ++t) w[t] += first * 64 + 16 * j;
    }
    __device__ __forceinline__ void next(int pitch, int64_t rows, int groups, uint32_t units, uint32_t inv)
    {
        const uint32_t bytes = chunk * 64 + 16 * (int)(threadIdx.x & 3) < pitch ? 16u : 0u;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            cp_async_16(to + t * 512, w[t], bytes);
            w[t] += by * 64;
        }
#pragma unroll
        for (int u = 0; u < 4 / GP; ++u) {
            const int g = scale_of((uint32_t)(chunk * (4 / GP) + u), units, inv);
            cp_async_4(to + to_scale + u * NT * 32, scale + (int64_t)g * rows, g < groups ? 4u : 0u);
        }
        chunk += by;
        to = to == to_first + (STAGES - 1) * Stage<NT, GP>::BYTES ? to_first : to + Stage<NT, GP>::BYTES;
    }
};
static_assert(8 * NT == 32, "a lane a column's scales");

__device__ __forceinline__ float activated(float g, int act)
{
    if (act == DSQ_SILU) return g / (1.f + expf(-g));
    const float u = 0.7978845608028654f * __fmaf_rn(0.044715f * g * g, g, g);
    return 0.5f * g * (1.f + tanhf(u));
}

// The same layer on 16 bits; arguments validated, p.w laid out for it.  gp: pieces of 32 codes that no group's end cuts.
DSQ_HIDDEN int run_wide(const MoeParams &p, int x_type, int gp_in, int gp_out, cudaStream_t s);

}  // namespace dsq_moe
