// Products of few rows with 4-bit weights that have a scale per group, on the 5th-generation
// tensor cores (dsq_wgemm_group.cu states the product and holds the kernel of small problems).
//
// The weights are the rows of an instruction, X its columns: D[128 weights' rows][rows of X]
// = A B^T with A the values 2 c + 1 (or c) of 128 rows of codes, made in registers and put
// into tensor memory, and B a few rows of X in shared memory.  A row of codes belongs to one
// thread, which makes its values, reads its sums of a group back and adds them, times the
// group's scale, to its totals in binary32 (one scale a thread and group).  An instruction of
// 128 x 16 x 16 does for 16 rows what 16 x 8 mma.sync tiles do with 16 times the operands'
// traffic through registers: at 8192 x 8192 with bf16 rows mma.sync took 23 us for one row and
// 64 us for 64, issue-bound.
//
//   * Four warps (a team) take a chunk of 128 codes of the block's 128 rows: codes from the
//     team's ring in shared memory (cp.async, each warp its own 32 rows), X of the chunk
//     from global memory through registers, permuted to the order in which codes come out of
//     their words, into the 128-byte swizzle.  A unit of 32 tensor-memory columns (64 codes
//     as 16-bit values, 128 as int8; less where a group ends sooner) is written while the
//     instructions of the unit before run: two buffers of A and of D a team.
//   * Teams of a block take its chunks in turn; blocks of a cluster share K and add their
//     totals through distributed shared memory.  All sums are in a fixed order.
//   * Exactly one block is on an SM (its shared memory sees to that): blocks of a cluster
//     wait for one another, and must not wait for tensor memory meanwhile.
//
// Every wait for the tensor core is bounded; where one runs out the outputs are NaN.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "dsq_groups.h"
#include "dsq_hooks.h"
#include "dsq_ptx.cuh"
#include "dsq_tc_host.h"
#include "dsq_types.cuh"
#include "dsq_wgemm_group.cuh"

using namespace dsq_ptx;

namespace {

__device__ __forceinline__ void tmem_st_32x8(uint32_t taddr, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr),
                 "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ void tmem_ld_32x8(uint32_t taddr, uint32_t (&r)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void st_cols(uint32_t at, const uint32_t (&r)[8]) { tmem_st_32x8(at, r); }
__device__ __forceinline__ void st_cols(uint32_t at, const uint32_t (&r)[16]) { tmem_st_32x16(at, r); }
__device__ __forceinline__ void st_cols(uint32_t at, const uint32_t (&r)[32]) { tmem_st_32x32(at, r); }
__device__ __forceinline__ void ld_cols(uint32_t at, uint32_t (&r)[8]) { tmem_ld_32x8(at, r); }
__device__ __forceinline__ void ld_cols(uint32_t at, uint32_t (&r)[16]) { tmem_ld_32x16(at, r); }
__device__ __forceinline__ void ld_cols(uint32_t at, uint32_t (&r)[32]) { tmem_ld_32x32(at, r); }

// COUNT instructions (32 bytes of K each) with A in tensor memory, issued by one elected lane of a
// converged warp; the first takes the accumulate flag.
#define DSQ_TS_1(KIND)                                                                                       \
    asm volatile("{\n\t.reg .pred p, pe;\n\t.reg .b64 d0;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 d0, {%2, %3};\n\t" \
                 "elect.sync _|pe, 0xffffffff;\n\t"                                                          \
                 "@pe tcgen05.mma.cta_group::1.kind::" KIND " [%0], [%1], d0, %4, p;\n\t}" ::"r"(d),          \
                 "r"(a), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)                                   \
                 : "memory")
#define DSQ_TS_2(KIND)                                                                                       \
    asm volatile("{\n\t.reg .pred p, q, pe;\n\t.reg .b64 d0, d1;\n\t.reg .b32 l1, a1;\n\t"                    \
                 "setp.ne.b32 p, %5, 0;\n\tsetp.eq.b32 q, %5, %5;\n\tadd.u32 l1, %2, 2;\n\tadd.u32 a1, %1, 8;\n\t" \
                 "mov.b64 d0, {%2, %3};\n\tmov.b64 d1, {l1, %3};\n\telect.sync _|pe, 0xffffffff;\n\t"          \
                 "@pe tcgen05.mma.cta_group::1.kind::" KIND " [%0], [%1], d0, %4, p;\n\t"                     \
                 "@pe tcgen05.mma.cta_group::1.kind::" KIND " [%0], [a1], d1, %4, q;\n\t}" ::"r"(d),          \
                 "r"(a), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)                                   \
                 : "memory")
#define DSQ_TS_4(KIND)                                                                                       \
    asm volatile("{\n\t.reg .pred p, q, pe;\n\t.reg .b64 d0, d1, d2, d3;\n\t.reg .b32 l1, l2, l3, a1, a2, a3;\n\t" \
                 "setp.ne.b32 p, %5, 0;\n\tsetp.eq.b32 q, %5, %5;\n\t"                                       \
                 "add.u32 l1, %2, 2;\n\tadd.u32 l2, %2, 4;\n\tadd.u32 l3, %2, 6;\n\t"                         \
                 "add.u32 a1, %1, 8;\n\tadd.u32 a2, %1, 16;\n\tadd.u32 a3, %1, 24;\n\t"                       \
                 "mov.b64 d0, {%2, %3};\n\tmov.b64 d1, {l1, %3};\n\tmov.b64 d2, {l2, %3};\n\tmov.b64 d3, {l3, %3};\n\t" \
                 "elect.sync _|pe, 0xffffffff;\n\t"                                                          \
                 "@pe tcgen05.mma.cta_group::1.kind::" KIND " [%0], [%1], d0, %4, p;\n\t"                     \
                 "@pe tcgen05.mma.cta_group::1.kind::" KIND " [%0], [a1], d1, %4, q;\n\t"                     \
                 "@pe tcgen05.mma.cta_group::1.kind::" KIND " [%0], [a2], d2, %4, q;\n\t"                     \
                 "@pe tcgen05.mma.cta_group::1.kind::" KIND " [%0], [a3], d3, %4, q;\n\t}" ::"r"(d),          \
                 "r"(a), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)                                   \
                 : "memory")
template <bool INT, int COUNT>
__device__ __forceinline__ void mma_ts_elect(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t b_hi, uint32_t idesc,
                                             uint32_t accumulate)
{
    static_assert(COUNT == 1 || COUNT == 2 || COUNT == 4, "instructions of a block");
    if constexpr (COUNT == 1) {
        if (INT) DSQ_TS_1("i8");
        else DSQ_TS_1("f16");
    } else if constexpr (COUNT == 2) {
        if (INT) DSQ_TS_2("i8");
        else DSQ_TS_2("f16");
    } else {
        if (INT) DSQ_TS_4("i8");
        else DSQ_TS_4("f16");
    }
}
#undef DSQ_TS_1
#undef DSQ_TS_2
#undef DSQ_TS_4

// once a wait has run out, instructions in flight get this long before their memory is given up
constexpr unsigned long long DRAIN_NS = 20000000ull;

// Bounded wait of all lanes of a warp; false where it ran out.
__device__ __noinline__ bool wait_slow(uint32_t bar, uint32_t parity, unsigned long long limit_ns)
{
    uint64_t t0, t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
    for (uint32_t it = 1;; ++it) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((it & 15u) == 0u) {
            asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
            if (t - t0 > limit_ns) return false;
        }
    }
}
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, unsigned long long limit_ns)
{
    bool ok = mbar_try_wait(bar, parity);
    if (!ok) ok = wait_slow(bar, parity, limit_ns);
    return __all_sync(~0u, ok);
}

// MC: columns of D that are read (rows of X); GP: pieces of 32 codes between two readings of D;
// TEAMS of four warps; STAGES of a team's ring
template <int XT, int MC, int GP, int TEAMS, int STAGES> struct Layout {
    static constexpr bool INT = XT == DSQ_I8;
    static constexpr int NC = MC < 16 ? 16 : MC;                  // columns of an instruction
    static constexpr int UC = INT ? 32 * GP : GP >= 2 ? 64 : 32;  // codes of a unit
    static constexpr int UNITS = 128 / UC;                        // of a chunk
    static constexpr int PER_FLUSH = 32 * GP / UC;
    static constexpr int AC = INT ? UC / 4 : UC / 2;              // tensor-memory columns of a unit
    static constexpr int A_COL = 2 * NC;                          // behind the two buffers of D
    static constexpr int TEAM_COLS = (2 * NC + 2 * AC + 31) / 32 * 32;
    static constexpr int COLS = TEAMS * TEAM_COLS <= 128 ? 128 : TEAMS * TEAM_COLS <= 256 ? 256 : 512;
    static constexpr int XBUF = NC * (INT ? 128 : 256);
    static constexpr int X_AT = 1024, RING_AT = X_AT + TEAMS * 2 * XBUF;
    static constexpr int STAGE = 128 * 64;
    static constexpr int BYTES = RING_AT + TEAMS * STAGES * STAGE + 1024;    // (its start is aligned to 1024)
    static constexpr int SUMS = TEAMS * MC * 512;
    static_assert(TEAMS * TEAM_COLS <= 512, "tensor memory");
    static_assert(BYTES <= 227 * 1024 && BYTES > 116 * 1024, "one block an SM");
    static_assert(SUMS <= TEAMS * STAGES * STAGE, "the sums take the rings' place");
};

template <int XT, int MC, int GP, int TEAMS, int STAGES>
__global__ void __launch_bounds__(TEAMS * 128, 1)
wgemm_group_tc_kernel(const DsqGroupGemm p, const int split, const unsigned long long wait_ns)
{
    using L = Layout<XT, MC, GP, TEAMS, STAGES>;
    constexpr bool INT = L::INT;
    constexpr int FLUSHES = 4 / GP;
    extern __shared__ uint8_t raw_smem[];
    const uint32_t smem = (smem_u32(raw_smem) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int team = warp >> 2, row = threadIdx.x & 127;         // row: of the block's 128
    const int tile = blockIdx.x / split, rank = blockIdx.x % split;
    const int64_t n0 = (int64_t)tile * 128;
    const int m0 = blockIdx.y * MC;
    const int rows = min(p.M - m0, MC);
    const int all = (p.K + 127) >> 7;
    const int c0 = (int)((int64_t)all * rank / split), c1 = (int)((int64_t)all * (rank + 1) / split);
    const int turns = c0 + team < c1 ? (c1 - c0 - team - 1) / TEAMS + 1 : 0;
    const uint32_t bars = smem + 16 + team * 16, slot = smem;
    const uint32_t xbuf = smem + L::X_AT + team * 2 * L::XBUF;
    const uint32_t ring = smem + L::RING_AT + team * STAGES * L::STAGE;

    if (warp == 0) {
        tmem_alloc(slot, L::COLS);
        tmem_relinquish();
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2 * TEAMS; ++i) mbar_init(smem + 16 + 8 * i, 1);
        mbar_init_fence();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = lds_32(slot) + team * L::TEAM_COLS;
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);    // this warp's 32 lanes

    // Copies of this warp's 32 rows of the team's next chunk: 16-byte piece j of a row's 64.  (Rows behind
    // the last are the last: their sums are not used.)
    const int j = lane & 3, mine = (warp & 3) * 32 + (lane >> 2);
    const uint8_t *src = p.W + n0 * p.pitch;
    const int last = (int)min((int64_t)127, p.N - 1 - n0);
    int row_at[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) row_at[k] = min(mine + 8 * k, last) * p.pitch;
    const uint32_t w_to = mine * 64 + ((j ^ (mine >> 1)) & 3) * 16;
    int w_left = turns, w_k = (c0 + team) * 64 + 16 * j;
    uint32_t w_stage = ring;
    auto issue_w = [&]() {
        if (w_left > 0) {
            const bool in = w_k < p.pitch;
            const uint8_t *s = src + (in ? w_k : 0);
            const uint32_t bytes = in ? 16u : 0u;
#pragma unroll
            for (int k = 0; k < 4; ++k) cp_async_16(w_stage + w_to + k * 512, s + row_at[k], bytes);
        }
        --w_left;
        w_k += TEAMS * 64;
        w_stage = w_stage == ring + (STAGES - 1) * L::STAGE ? ring : w_stage + L::STAGE;
        cp_async_commit();
    };
    // X of a chunk: 16-byte pieces of its rows, spread over the team: piece pc of rows r0, r0 + RS, ...
    constexpr int PIECES = INT ? 8 : 16, RS = 128 / PIECES, XP = (MC + RS - 1) / RS;
    constexpr int ELEMENT = INT ? 1 : 2;
    const int pc = row % PIECES, r0 = row / PIECES;
    const uint8_t *xsrc = p.X + ((int64_t)(m0 + r0) * p.K) * ELEMENT + 16 * pc;
    const int64_t x_step = (int64_t)RS * p.K * ELEMENT;
    const uint32_t x_to = xbuf + (pc >> 3) * (L::NC * 128) + r0 * 128 + (((pc & 7) ^ (r0 & 7)) << 4);
    static_assert(RS % 8 == 0, "the swizzle of a thread's rows is one");
    uint4 x[XP];
    float sc[FLUSHES];
    int l_left = turns, l_chunk = c0 + team;
    auto load = [&]() {
        const int k_at = l_chunk * (PIECES * 16);                 // bytes into the row
        const bool in = l_left > 0 && k_at + 16 * pc < p.K * ELEMENT;
        const uint8_t *s = xsrc + (in ? k_at : 0);
#pragma unroll
        for (int k = 0; k < XP; ++k, s += x_step) {
            x[k] = make_uint4(0u, 0u, 0u, 0u);
            if (in && r0 + k * RS < rows) x[k] = __ldg(reinterpret_cast<const uint4 *>(s));
        }
#pragma unroll
        for (int f = 0; f < FLUSHES; ++f) {
            const int g = p.group_of((uint32_t)(l_chunk * FLUSHES + f));
            sc[f] = 0.f;
            if (l_left > 0 && g < p.groups && row <= last) sc[f] = __ldg(p.scales + (int64_t)g * p.N + n0 + row);
        }
        --l_left;
        l_chunk += TEAMS;
    };

    grid_dependency_wait();
    grid_launch_dependents();
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) issue_w();
    load();

    float total[MC];
#pragma unroll
    for (int i = 0; i < MC; ++i) total[i] = 0.f;
    const uint32_t idesc = INT ? idesc_i8(L::NC, true, true) : (XT == DSQ_BF16 ? idesc_bf16(L::NC) : dsq_idesc_f16(L::NC));
    const uint32_t base = dsq_value_base<XT>(p.odd);
    const uint32_t one = p.odd ? 0x08080808u : 0u;
    bool ok = true;
    uint32_t unit = 0, flush = 0;             // of the team so far
    float pending = 0.f;                      // scale of the sums that wait in D
    uint32_t r_stage = ring;

    // every phase of a barrier is waited for by every thread before the next can end
    auto wait_unit = [&](uint32_t u) {
        ok = wait_warp(bars + 8 * (u & 1), (u >> 1) & 1, ok ? wait_ns : 0) && ok;
    };
    // D of flush `f`, whose instructions are done: the totals take it
    auto take = [&](uint32_t f, float s) {
        tc_fence_after_sync();
        const uint32_t d = lanes + (f & 1) * L::NC;
        constexpr int STEP = MC < 32 ? MC : 32;
#pragma unroll
        for (int h = 0; h < MC / STEP; ++h) {
            uint32_t v[STEP];
            ld_cols(d + h * STEP, v);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < STEP; ++i)
                total[h * STEP + i] = __fmaf_rn(INT ? (float)(int)v[i] : __uint_as_float(v[i]), s, total[h * STEP + i]);
        }
    };

#pragma unroll 1
    for (int i = 0; i < turns; ++i) {
        cp_async_wait<STAGES - 2>();
        __syncwarp();             // the chunk's codes are here, and those of the last one have been read
        issue_w();
        // X: the instructions of the chunk before the last, which read this buffer, are done
        const uint32_t xb = xbuf + (i & 1) * L::XBUF;
#pragma unroll
        for (int k = 0; k < XP; ++k) {
            if (r0 + k * RS < rows) {
                const uint4 v = x[k];
                const uint32_t to = x_to + (i & 1) * L::XBUF + k * (RS * 128);
                if (INT)
                    sts_128(to, __byte_perm(v.x, v.y, 0x6420), __byte_perm(v.x, v.y, 0x7531),
                            __byte_perm(v.z, v.w, 0x6420), __byte_perm(v.z, v.w, 0x7531));
                else
                    sts_128(to, __byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632),
                            __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
            }
        }
        fence_proxy_async_smem();
        float now[FLUSHES];
#pragma unroll
        for (int f = 0; f < FLUSHES; ++f) now[f] = sc[f];
        load();
        const uint32_t codes = r_stage + row * 64;
        r_stage = r_stage == ring + (STAGES - 1) * L::STAGE ? ring : r_stage + L::STAGE;
#pragma unroll
        for (int u = 0; u < L::UNITS; ++u, ++unit) {
            // the values of this row's codes
            uint32_t a[L::AC];
#pragma unroll
            for (int q = 0; q < L::UC / 32; ++q) {
                const int pc = u * (L::UC / 32) + q;              // 16-byte piece of the row
                const uint4 w4 = lds_128(codes + ((pc ^ (row >> 1)) & 3) * 16);
                const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if constexpr (INT) {
                        a[8 * q + 2 * k] = ((w[k] << 4) & 0xF0F0F0F0u) | one;
                        a[8 * q + 2 * k + 1] = (w[k] & 0xF0F0F0F0u) | one;
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) a[16 * q + 4 * k + e] = dsq_value_pair<XT>(w[k], e, base);
                    }
                }
            }
            if (unit >= 2) wait_unit(unit - 2);
            st_cols(lanes + L::A_COL + (unit & 1) * L::AC, a);
            tmem_st_wait();
            tc_fence_before_sync();
            named_barrier_sync(1 + team, 128);
            if ((warp & 3) == 0) {
                tc_fence_after_sync();
                const int at = u * L::UC * (INT ? 1 : 2);         // bytes into the chunk's rows
                const uint64_t desc = smem_desc_sw128(xb + (at >> 7) * (L::NC * 128) + (at & 127));
                const uint32_t d = tmem + (flush & 1) * L::NC;
                mma_ts_elect<INT, L::AC / 8>(d, tmem + L::A_COL + (unit & 1) * L::AC, (uint32_t)desc,
                                             (uint32_t)(desc >> 32), idesc, u % L::PER_FLUSH);
                mma_commit_elect(bars + 8 * (unit & 1));
                __syncwarp();
            }
            // the sums before this unit's flush, while its instructions run
            if (u % L::PER_FLUSH == L::PER_FLUSH - 1) {
                if (flush) {
                    // (that flush ended PER_FLUSH units ago; two: this unit's A has waited for it)
                    if (L::PER_FLUSH == 1) wait_unit(unit - 1);
                    take(flush - 1, pending);
                }
                pending = now[u / L::PER_FLUSH];
                ++flush;
            }
        }
    }
    if (flush) {
        wait_unit(unit - 1);
        if (!ok) wait_warp(bars + 8 * ((unit - 1) & 1), ((unit - 1) >> 1) & 1, DRAIN_NS);
        take(flush - 1, pending);
    }
    cp_async_wait<0>();
    tc_fence_before_sync();
    const int failed = __syncthreads_or(!ok);
    if (warp == 0) {
        tc_fence_after_sync();
        tmem_dealloc(lds_32(slot), L::COLS);
    }
    // the teams' totals, [team][column][row], added in turn; then those of the cluster's blocks
    const uint32_t sums = smem + L::RING_AT;
#pragma unroll
    for (int i = 0; i < MC; ++i)
        sts_32(sums + ((team * MC + i) * 128 + row) * 4, __float_as_uint(total[i]));
    __syncthreads();
    const float unit_value = dsq_value_unit<XT>(p.odd);
    for (int m = team; m < rows; m += TEAMS) {
        float s = 0.f;
#pragma unroll
        for (int t = 0; t < TEAMS; ++t) s += __uint_as_float(lds_32(sums + ((t * MC + m) * 128 + row) * 4));
        if (failed) s = __uint_as_float(0x7FC00000u);
        if (split == 1) {
            if (n0 + row < p.N) p.store(m0 + m, n0 + row, s * unit_value);
        } else {
            sts_32(sums + (m * 128 + row) * 4, __float_as_uint(s));
        }
    }
    if (split > 1) {
        cluster_sync_all();
        for (int m = rank + team * split; m < rows; m += TEAMS * split) {
            float s = 0.f;
            for (int r = 0; r < split; ++r) s += __uint_as_float(ld_cluster_32(map_to_cta(sums + (m * 128 + row) * 4, r)));
            if (n0 + row < p.N) p.store(m0 + m, n0 + row, s * unit_value);
        }
        cluster_sync_all();       // nobody leaves while its sums are read
    }
}

template <int XT, int MC, int GP, int TEAMS, int STAGES>
int launch(const DsqGroupGemm &p, cudaStream_t s)
{
    using L = Layout<XT, MC, GP, TEAMS, STAGES>;
    static std::atomic<unsigned long long> configured{0};
    const auto kernel = wgemm_group_tc_kernel<XT, MC, GP, TEAMS, STAGES>;
    const int st = dsq_allow_smem((const void *)kernel, L::BYTES, &configured);
    if (st) return st;
    const int64_t tiles = (p.N + 127) / 128, mt = (p.M + MC - 1) / MC;
    const int chunks = (p.K + 127) / 128, sms = dsq_sm_count() > 0 ? dsq_sm_count() : 148;
    // Blocks along K: the time of a wave is its chunks a team and about six more for the start
    // and the end of a block.
    int split = 1;
    double best = 1e30;
    for (int c = 1; c <= 8 && c <= chunks; c *= 2) {
        const double waves = (double)((tiles * mt * c + sms - 1) / sms);
        const double t = waves * ((double)((chunks + c - 1) / c + TEAMS - 1) / TEAMS + 6.0 + (c > 1 ? 1.0 : 0.0));
        if (t < best) {
            best = t;
            split = c;
        }
    }
    if (tiles * split > 0x7FFFFFFF || mt > 65535) return DSQ_ERR_SIZE;
    const DsqLaunchHooks h = dsq_launch_hooks();
    return dsq_launch(kernel, dim3((unsigned)(tiles * split), (unsigned)mt), dim3(TEAMS * 128), (size_t)L::BYTES, s,
                      h.pdl, split, p, split, h.wait_ns);
}

template <int XT, int GP> int pick(const DsqGroupGemm &p, cudaStream_t s)
{
    if (p.M <= 8) return launch<XT, 8, GP, 4, 4>(p, s);
    if (p.M <= 16) return launch<XT, 16, GP, 4, 4>(p, s);
    if (p.M <= 32) return launch<XT, 32, GP, 3, 4>(p, s);
    return launch<XT, 64, GP, 2, 6>(p, s);
}

template <int XT> int pick_group(DsqGroupGemm p, int64_t group, cudaStream_t s)
{
    const int gp = dsq_group_pieces(group);
    p.set_units(group, gp);
    return gp == 4 ? pick<XT, 4>(p, s) : gp == 2 ? pick<XT, 2>(p, s) : pick<XT, 1>(p, s);
}

}  // namespace

int dsq_wgemm_group_tc(const DsqGroupGemm &p, int x_type, int64_t group, cudaStream_t s)
{
    switch (x_type) {
    case DSQ_BF16: return pick_group<DSQ_BF16>(p, group, s);
    case DSQ_F16: return pick_group<DSQ_F16>(p, group, s);
    default: return pick_group<DSQ_I8>(p, group, s);
    }
}
