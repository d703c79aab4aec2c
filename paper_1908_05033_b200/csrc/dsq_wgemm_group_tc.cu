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
//   * TEAMS of four warps take the block's chunks of 128 codes of 128 rows in turn, two at a time: codes
//     from the team's ring in shared memory (cp.async, each warp its own 32 rows, whole lines of 128
//     bytes: with 64 of a line at a time memory gave 1.6 TB/s), X of a chunk from global memory
//     through registers, permuted to the order in which codes come out of their words, into the
//     128-byte swizzle.  One warp of the team issues the instructions.
//   * Four more warps take the sums: a chunk's (a group's, where groups end sooner) lie in one of the
//     team's places in tensor memory; they read them, give the place back and add.  Making values and
//     adding sums are both bound by issue slots and by latencies, and with the totals out of the
//     teams' registers 16 warps fit (two teams that did both took 34 us for 64 rows at 8192 x 8192).
//   * Blocks of a cluster share K and add their totals through distributed shared memory, in order.
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

__device__ __forceinline__ void tmem_ld_32x8(uint32_t taddr, uint32_t (&r)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr)
                 : "memory");
}
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

// loads that stay where they stand: a turn ahead of their use
__device__ __forceinline__ uint4 load_ahead(const uint8_t *p)
{
    uint4 v;
    asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ void cp_async_4(uint32_t dst, const float *src)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

// once a wait has run out, instructions in flight get this long before their memory is given up
constexpr unsigned long long DRAIN_NS = 20000000ull;

// Bounded wait of all lanes of a warp; false where it ran out.
__device__ __noinline__ bool wait_slow(uint32_t bar, uint32_t parity, unsigned long long limit_ns)
{
    uint64_t t0, t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
    for (uint32_t it = 1;; ++it) {
        if (mbar_try_wait(bar, parity, 20u)) return true;
        if ((it & 15u) == 0u) {
            asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
            if (t - t0 > limit_ns) return false;
        }
    }
}
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, unsigned long long limit_ns)
{
    bool ok = mbar_try_wait(bar, parity, 20u);
    if (!ok) ok = wait_slow(bar, parity, limit_ns);
    return __all_sync(~0u, ok);
}

constexpr int AHEAD = 8;          // chunks whose scales are on their way
// MC: columns of D that are read (rows of X); GP: pieces of 32 codes of a sum
template <int XT, int MC, int GP, int TEAMS, int STAGES> struct Layout {
    static constexpr bool INT = XT == DSQ_I8;
    static constexpr int NC = MC < 16 ? 16 : MC;                  // columns of an instruction
    static constexpr int FLUSHES = 4 / GP;                        // sums of a chunk
    static constexpr int AC = INT ? 32 : 64;                      // tensor-memory columns of a chunk's values
    // places of a team for its sums (a power of two): the phases of a place's barriers are waited for in
    // order by the team's issuing warp, so no two teams share one
    static constexpr int ABUF = TEAMS * (2 * AC + NC) <= 512 ? 2 : 1;         // buffers of a team's values
    static constexpr int ROOM = (512 - TEAMS * ABUF * AC) / (TEAMS * NC), PLACES = ROOM >= 4 ? 4 : ROOM >= 2 ? 2 : 1;
    static constexpr int SLOTS = TEAMS * PLACES;
    static constexpr int A_COL = SLOTS * NC;
    static constexpr int USED = A_COL + TEAMS * ABUF * AC;
    static constexpr int COLS = USED <= 128 ? 128 : USED <= 256 ? 256 : 512;
    static constexpr int XBUF = NC * (INT ? 128 : 256);
    static constexpr int X_AT = 1024, RING_AT = X_AT + TEAMS * 2 * XBUF;
    static constexpr int STAGE = 128 * 128;                       // two chunks
    static constexpr int S_AT = RING_AT + TEAMS * STAGES * STAGE, S_STAGE = FLUSHES * 512;    // scales of a chunk
    static constexpr int BYTES = S_AT + AHEAD * S_STAGE + 1024;              // (its start is aligned to 1024)
    static constexpr int THREADS = (TEAMS + 1) * 128;
    // barriers: sums ready and place free of each slot, values read of each team
    static constexpr int READY = 16, FREE = READY + 8 * SLOTS, READ = FREE + 8 * SLOTS;
    static_assert(ROOM >= 1 && USED <= 512 && READ + 16 * TEAMS <= X_AT, "tensor memory");
    static_assert(BYTES <= 227 * 1024 && BYTES > 116 * 1024, "one block an SM");
    static_assert(MC * 512 <= TEAMS * STAGES * STAGE, "the totals take the rings' place");
};

template <int XT, int MC, int GP, int TEAMS, int STAGES>
__global__ void __launch_bounds__((TEAMS + 1) * 128, 1)
wgemm_group_tc_kernel(const DsqGroupGemm p, const int split, const unsigned long long wait_ns)
{
    using L = Layout<XT, MC, GP, TEAMS, STAGES>;
    constexpr bool INT = L::INT;
    constexpr int FLUSHES = L::FLUSHES;
    extern __shared__ uint8_t raw_smem[];
    const uint32_t smem = (smem_u32(raw_smem) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int team = warp >> 2, row = threadIdx.x & 127;         // row: of the block's 128
    const int tile = blockIdx.x / split, rank = blockIdx.x % split;
    const int64_t n0 = (int64_t)tile * 128;
    const int m0 = blockIdx.y * MC;
    const int rows = min(p.M - m0, MC);
    const int all = (p.K + 127) >> 7;
    // whole pairs of chunks to a block
    const int pairs = (all + 1) >> 1, c0 = 2 * (int)((int64_t)pairs * rank / split);
    const int chunks = min(2 * (int)((int64_t)pairs * (rank + 1) / split), all) - c0;
    const int last = (int)min((int64_t)127, p.N - 1 - n0);       // row of weights of this block

    if (warp == 0) {
        tmem_alloc(smem, L::COLS);
        tmem_relinquish();
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < L::SLOTS; ++i) {
            mbar_init(smem + L::READY + 8 * i, 1);
            mbar_init(smem + L::FREE + 8 * i, 4);
        }
        for (int i = 0; i < 2 * TEAMS; ++i) mbar_init(smem + L::READ + 8 * i, 1);
        mbar_init_fence();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = lds_32(smem);
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);    // this warp's 32 lanes
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity) { ok = wait_warp(smem + bar, parity, ok ? wait_ns : 0) && ok; };
    grid_dependency_wait();
    grid_launch_dependents();

    float total[MC];                                             // (of the last team's threads)
#pragma unroll
    for (int i = 0; i < MC; ++i) total[i] = 0.f;
    if (team < TEAMS) {
        const uint32_t xbuf = smem + L::X_AT + team * 2 * L::XBUF;
        const uint32_t ring = smem + L::RING_AT + team * STAGES * L::STAGE;
        // the team's chunks: c0 + 2 (team + TEAMS i) and the one behind it
        const int my_pairs = 2 * team < chunks ? ((chunks + 1) / 2 - team - 1) / TEAMS + 1 : 0;
        const int turns = my_pairs == 0 ? 0 : 2 * my_pairs - ((chunks & 1) && (chunks / 2) % TEAMS == team);
        // Copies of this warp's 32 rows of the team's next two chunks: 16-byte piece j of a row's 128.  (Rows
        // behind the last are the last: their sums are not used.)
        const int j = lane & 7, mine = (warp & 3) * 32 + (lane >> 3);
        const uint8_t *src = p.W + n0 * p.pitch;
        int row_at[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) row_at[k] = min(mine + 4 * k, last) * p.pitch;
        const uint32_t w_to = mine * 128;
        int w_left = my_pairs, w_k = (c0 + 2 * team) * 64 + 16 * j;
        uint32_t w_stage = ring;
        auto issue_w = [&]() {
            if (w_left > 0) {
                const bool in = w_k < p.pitch;
                const uint8_t *s = src + (in ? w_k : 0);
                const uint32_t bytes = in ? 16u : 0u;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    cp_async_16(w_stage + w_to + k * 512 + ((j ^ (mine + 4 * k)) & 7) * 16, s + row_at[k], bytes);
            }
            --w_left;
            w_k += TEAMS * 128;
            w_stage = w_stage == ring + (STAGES - 1) * L::STAGE ? ring : w_stage + L::STAGE;
            cp_async_commit();
        };
        // X of a chunk: 16-byte pieces of its rows, spread over the team: piece pc of rows r0, r0 + RS, ...
        constexpr int PIECES = INT ? 8 : 16, RS = 128 / PIECES, XP = (MC + RS - 1) / RS;
        constexpr int ELEMENT = INT ? 1 : 2;
        const int pc = row % PIECES, r0 = row / PIECES;
        // (rows behind the last are the last: their columns of D are not read)
        const uint8_t *xsrc = p.X + (int64_t)m0 * p.K * ELEMENT + 16 * pc;
        uint32_t x_at[XP];
#pragma unroll
        for (int k = 0; k < XP; ++k) x_at[k] = (uint32_t)min(r0 + k * RS, rows - 1) * (uint32_t)(p.K * ELEMENT);
        const uint32_t x_to = xbuf + (pc >> 3) * (L::NC * 128) + r0 * 128 + (((pc & 7) ^ (r0 & 7)) << 4);
        static_assert(RS % 8 == 0 && XP * RS <= L::NC, "the swizzle of a thread's rows is one");
        uint4 x[XP];
        int l_turn = 0, l_k = (c0 + 2 * team) * (PIECES * 16);   // bytes into the row
        auto load_x = [&]() {
            if (l_turn < turns && l_k + 16 * pc < p.K * ELEMENT) {
                const uint8_t *s = xsrc + l_k;
#pragma unroll
                for (int k = 0; k < XP; ++k) x[k] = load_ahead(s + x_at[k]);
            } else {
#pragma unroll
                for (int k = 0; k < XP; ++k) x[k] = make_uint4(0u, 0u, 0u, 0u);
            }
            l_k += (l_turn & 1 ? 2 * TEAMS - 1 : 1) * (PIECES * 16);
            ++l_turn;
        };
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s) issue_w();
        load_x();
        const uint32_t idesc = INT ? idesc_i8(L::NC, true, true) : (XT == DSQ_BF16 ? idesc_bf16(L::NC) : dsq_idesc_f16(L::NC));
        const uint32_t base = dsq_value_base<XT>(p.odd), one = p.odd ? 0x08080808u : 0u;
        // instructions of the team's chunk i have read its values and X
        auto wait_read = [&](int i) { wait(L::READ + 16 * team + 8 * (i % L::ABUF), (i / L::ABUF) & 1); };
        uint32_t r_stage = ring;
#pragma unroll 1
        for (int i = 0; i < turns; ++i) {
            if ((i & 1) == 0) {
                cp_async_wait<STAGES - 2>();
                __syncwarp();     // the two chunks' codes are here, and those before them have been read
                issue_w();
            }
            // (X has two buffers too: its last chunk but one has been waited for)
            if (L::ABUF == 2 && i >= 2) wait_read(i - 2);
            const uint32_t a_col = L::A_COL + (team * L::ABUF + i % L::ABUF) * L::AC;
#pragma unroll
            for (int k = 0; k < XP; ++k) {
                const uint4 v = x[k];
                const uint32_t to = x_to + (i & 1) * L::XBUF + k * (RS * 128);
                if (INT)
                    sts_128(to, __byte_perm(v.x, v.y, 0x6420), __byte_perm(v.x, v.y, 0x7531),
                            __byte_perm(v.z, v.w, 0x6420), __byte_perm(v.z, v.w, 0x7531));
                else
                    sts_128(to, __byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632),
                            __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
            }
            fence_proxy_async_smem();
            load_x();
            const uint32_t codes = r_stage + row * 128;
            if (i & 1) r_stage = r_stage == ring + (STAGES - 1) * L::STAGE ? ring : r_stage + L::STAGE;
            // the values of this row's codes, 32 columns at a time
#pragma unroll
            for (int h = 0; h < L::AC / 32; ++h) {
                constexpr int P16 = INT ? 4 : 2;                  // 16-byte pieces of the row
                uint32_t a[32];
#pragma unroll
                for (int q = 0; q < P16; ++q) {
                    const uint4 w4 = lds_128(codes + (((4 * (i & 1) + P16 * h + q) ^ row) & 7) * 16);
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
                if (L::ABUF == 1 && h == 0 && i > 0) wait_read(i - 1);
                tmem_st_32x32(lanes + a_col + 32 * h, a);
            }
            tmem_st_wait();
            tc_fence_before_sync();
            named_barrier_sync(1 + team, 128);
            if ((warp & 3) == 0) {
                const uint64_t desc = smem_desc_sw128(xbuf + (i & 1) * L::XBUF);
                const uint32_t hi = (uint32_t)(desc >> 32);
#pragma unroll
                for (int f = 0; f < FLUSHES; ++f) {
                    const uint32_t use = i * FLUSHES + f, slot = team * L::PLACES + use % L::PLACES;
                    if (use >= L::PLACES) wait(L::FREE + 8 * slot, ((use / L::PLACES) & 1) ^ 1);
                    tc_fence_after_sync();
                    constexpr int COUNT = L::AC / 8 / FLUSHES, BLOCK = COUNT < 4 ? COUNT : 4;
#pragma unroll
                    for (int b = 0; b < COUNT / BLOCK; ++b) {
                        const int at = (f * COUNT + b * BLOCK) * 32;          // bytes into the chunk's rows
                        mma_ts_elect<INT, BLOCK>(tmem + slot * L::NC, tmem + a_col + (f * COUNT + b * BLOCK) * 8,
                                                 (uint32_t)desc + (((at >> 7) * (L::NC * 128) + (at & 127)) >> 4), hi, idesc, b);
                    }
                    mma_commit_elect(smem + L::READY + 8 * slot);
                }
                mma_commit_elect(smem + L::READ + 16 * team + 8 * (i % L::ABUF));
                __syncwarp();
            }
        }
        // the last instructions read X and the values to the end
        for (int i = max(0, turns - L::ABUF); i < turns; ++i) {
            wait_read(i);
            if (!ok) wait_warp(smem + L::READ + 16 * team + 8 * (i % L::ABUF), (i / L::ABUF) & 1, DRAIN_NS);
        }
    } else {
        // A row's scales go through a ring of their own, each thread's copies for itself.  (A chunk ahead, in
        // registers, the wait for them was the kernel's time: 32 times 0.6 us.)
        const uint32_t s_ring = smem + L::S_AT + row * 4;
        const float *scales = p.scales + n0 + min(row, last);
        auto issue_s = [&](int c) {
            if (c < chunks) {
#pragma unroll
                for (int f = 0; f < FLUSHES; ++f) {
                    const int g = min(p.group_of((uint32_t)((c0 + c) * FLUSHES + f)), p.groups - 1);
                    cp_async_4(s_ring + (c % AHEAD) * L::S_STAGE + f * 512, scales + (int64_t)g * p.N);
                }
            }
            cp_async_commit();
        };
#pragma unroll 1
        for (int c = 0; c < AHEAD - 1; ++c) issue_s(c);
        uint32_t of = 0, turn = 0;                               // the chunk's team, and its turn there
#pragma unroll 1
        for (int i = 0; i < chunks; ++i) {
            cp_async_wait<AHEAD - 2>();
            float now[FLUSHES];
#pragma unroll
            for (int f = 0; f < FLUSHES; ++f)
                now[f] = __uint_as_float(lds_32(s_ring + (i % AHEAD) * L::S_STAGE + f * 512));
            issue_s(i + AHEAD - 1);
#pragma unroll
            for (int f = 0; f < FLUSHES; ++f) {
                const uint32_t use = turn * FLUSHES + f, slot = of * L::PLACES + use % L::PLACES;
                wait(L::READY + 8 * slot, (use / L::PLACES) & 1);
                tc_fence_after_sync();
                constexpr int STEP = MC < 32 ? MC : 32;
#pragma unroll
                for (int h = 0; h < MC / STEP; ++h) {
                    uint32_t v[STEP];
                    ld_cols(lanes + slot * L::NC + h * STEP, v);
                    tmem_ld_wait();
                    if (h == MC / STEP - 1) {                     // the place is free again
                        tc_fence_before_sync();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem + L::FREE + 8 * slot);
                    }
#pragma unroll
                    for (int e = 0; e < STEP; ++e)
                        total[h * STEP + e] = __fmaf_rn(INT ? (float)(int)v[e] : __uint_as_float(v[e]), now[f],
                                                        total[h * STEP + e]);
                }
            }
            if ((i & 1) == 0) {
                ++turn;
            } else if (++of == TEAMS) {
                of = 0;
                ++turn;
            } else {
                --turn;
            }
        }
    }
    cp_async_wait<0>();
    tc_fence_before_sync();
    const int failed = __syncthreads_or(!ok);
    if (warp == 0) {
        tc_fence_after_sync();
        tmem_dealloc(lds_32(smem), L::COLS);
    }
    if (split == 1) {
        if (team == TEAMS && row <= last) {
            const float unit = failed ? __uint_as_float(0x7FC00000u) : dsq_value_unit<XT>(p.odd);
#pragma unroll
            for (int m = 0; m < MC; ++m)
                if (m < rows) p.store(m0 + m, n0 + row, total[m] * unit);
        }
        return;
    }
    // the totals of the cluster's blocks, [row of X][row of weights], added in their order
    const uint32_t sums = smem + L::RING_AT;
    if (team == TEAMS) {
#pragma unroll
        for (int m = 0; m < MC; ++m)
            sts_32(sums + (m * 128 + row) * 4, failed ? 0x7FC00000u : __float_as_uint(total[m]));
    }
    cluster_sync_all();
    const float unit = dsq_value_unit<XT>(p.odd);
    for (int m = rank + team * split; m < rows; m += (TEAMS + 1) * split) {
        float s = 0.f;
        for (int r = 0; r < split; ++r) s += __uint_as_float(ld_cluster_32(map_to_cta(sums + (m * 128 + row) * 4, r)));
        if (row <= last) p.store(m0 + m, n0 + row, s * unit);
    }
    cluster_sync_all();           // nobody leaves while its sums are read
}

// Clusters of `split` blocks that run at once (a GPC's SMs bound them: of eight blocks fewer than 148 / 8).
template <class K> int active_clusters(K kernel, int split, int threads, int bytes, std::atomic<int> *cached)
{
    int n = cached->load(std::memory_order_relaxed);
    if (n > 0) return n;
    const int sms = dsq_sm_count() > 0 ? dsq_sm_count() : 148;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(split * sms));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)bytes;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n <= 0) {
        cudaGetLastError();
        n = sms / split;
    }
    cached->store(n, std::memory_order_relaxed);
    return n;
}

// est_us: the launch's estimated time is written there and nothing is launched
template <int XT, int MC, int GP, int TEAMS, int STAGES>
int launch(const DsqGroupGemm &p, cudaStream_t s, double *est_us)
{
    using L = Layout<XT, MC, GP, TEAMS, STAGES>;
    static std::atomic<unsigned long long> configured{0};
    static std::atomic<int> active[4];
    const auto kernel = wgemm_group_tc_kernel<XT, MC, GP, TEAMS, STAGES>;
    const int st = dsq_allow_smem((const void *)kernel, L::BYTES, &configured);
    if (st) return st;
    const int64_t tiles = (p.N + 127) / 128, mt = (p.M + MC - 1) / MC;
    const int pairs = ((p.K + 127) / 128 + 1) / 2, sms = dsq_sm_count() > 0 ? dsq_sm_count() : 148;
    // Blocks along K.  us of a wave: 3.6 for its start and end, the cluster's sums 1.0, and a turn of a
    // team: measured at 8192 x 8192 (11 turns): 18.8, 21.7 and 31.8 us for 16, 32 and 64 rows, int8 14.5,
    // 16.8 and 21.4.
    constexpr double TURN = XT == DSQ_I8 ? (MC <= 16 ? 0.9 : MC <= 32 ? 1.1 : 1.5) : (MC <= 16 ? 1.3 : MC <= 32 ? 1.55 : 2.5);
    int split = 1;
    double best = 1e30;
    for (int c = 1, k = 0; c <= 8 && c <= pairs; c *= 2, ++k) {
        const int64_t at_once = c == 1 ? sms : active_clusters(kernel, c, L::THREADS, L::BYTES, &active[k]);
        const double waves = (double)((tiles * mt + at_once - 1) / at_once);
        const int turns = 2 * (((pairs + c - 1) / c + TEAMS - 1) / TEAMS);
        const double t = waves * (3.6 + TURN * turns + (c > 1 ? 1.0 : 0.0));
        if (t < best) {
            best = t;
            split = c;
        }
    }
    if (est_us) {
        *est_us = best;
        return DSQ_OK;
    }
    if (tiles * split > 0x7FFFFFFF || mt > 65535) return DSQ_ERR_SIZE;
    const DsqLaunchHooks h = dsq_launch_hooks();
    return dsq_launch(kernel, dim3((unsigned)(tiles * split), (unsigned)mt), dim3(L::THREADS), (size_t)L::BYTES, s,
                      h.pdl, split, p, split, h.wait_ns);
}

template <int XT, int GP> int pick(const DsqGroupGemm &p, cudaStream_t s, double *est_us)
{
    if (p.M <= 8) return launch<XT, 8, GP, 3, 3>(p, s, est_us);
    if (p.M <= 16) return launch<XT, 16, GP, 3, 3>(p, s, est_us);
    if (p.M <= 32) return launch<XT, 32, GP, 3, 3>(p, s, est_us);
    return launch<XT, 64, GP, 3, 2>(p, s, est_us);
}

template <int XT> int pick_group(DsqGroupGemm p, int64_t group, cudaStream_t s, double *est_us)
{
    const int gp = dsq_group_pieces(group);
    p.set_units(group, gp);
    return gp == 4 ? pick<XT, 4>(p, s, est_us) : gp == 2 ? pick<XT, 2>(p, s, est_us) : pick<XT, 1>(p, s, est_us);
}

}  // namespace

int dsq_wgemm_group_tc(const DsqGroupGemm &p, int x_type, int64_t group, cudaStream_t s, double *est_us)
{
    switch (x_type) {
    case DSQ_BF16: return pick_group<DSQ_BF16>(p, group, s, est_us);
    case DSQ_F16: return pick_group<DSQ_F16>(p, group, s, est_us);
    default: return pick_group<DSQ_I8>(p, group, s, est_us);
    }
}
