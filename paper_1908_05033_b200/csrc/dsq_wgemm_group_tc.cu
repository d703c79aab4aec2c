// Products of few rows with 4-bit weights that have a scale per group, on the 5th-generation
// tensor cores (dsq_wgemm_group.cu states the product and holds the kernel of small problems).
//
// The weights are the rows of an instruction, X its columns: D[128 weights' rows][rows of X]
// = A B^T with A the values of 128 rows of codes, made in registers and put into tensor memory,
// and B a few rows of X in shared memory.  A row of codes belongs to one thread of those that make
// values and to one of those that read its sums of a group back and add them, times the group's
// scale, to its totals in binary32.  An instruction of 128 x 16 x 16 does for 16 rows what 16 x 8
// mma.sync tiles do with 16 times the operands' traffic through registers: at 8192 x 8192 with bf16
// rows mma.sync takes 16.0 us for 8 rows, 21 for 16, 30 for 32 and 64 for 64.
//
//   * One warp copies: a stage of the ring is two chunks of 128 codes of 128 rows (whole lines of 128
//     bytes) and X's elements for them, both by TMA into the 128-byte swizzle; zeros behind the ends.
//   * TEAMS of four warps make values, chunks in turn: 64 columns of tensor memory a chunk for 16-bit
//     rows, 32 for 8-bit ones.  Three operations for two 16-bit values, in the order of X.  (With pairs as
//     they come out of a word, codes i and i + 4, X had to be permuted on its way, in the same warps:
//     that cost 64 rows 31.8 us where they now take 20.1.)
//   * Two warps issue the instructions, chunks in turn, with an elected lane.  (One thread in a branch of its
//     own took 75 cycles an instruction and 200 a commit, an elected lane of a whole warp 30 and 40: 8 rows
//     17.4 against 15.4 us.  One issuing warp instead of two: 22.)
//   * One, two or four teams more take the sums: a chunk's (a group's, where groups end sooner) lie in
//     one of the places in tensor memory; they read them, give the place back and add.
//   * Blocks of a cluster share K and add their totals through distributed shared memory, in order.
//   * Exactly one block is on an SM (its shared memory sees to that): blocks of a cluster
//     wait for one another, and must not wait for tensor memory meanwhile.
//
// Bound at 8192 x 8192, 16 rows of bf16 (16.4 us; codes alone 5.3 us at the copy's rate): 3.8 us of
// launch, set-up and the cluster's sums, 7 for the copies and the roles' signals to one another with no
// work between them, the rest unpacking and instructions, of which no pipe is full (issue slots 47 %,
// ALU 44 %, tensor 6 %).  64 rows 20.2, in 8 bits 18.5; 8 rows 15.4 and 12.9; groups of 32 instead of 128, 16 rows:
// 21.6 us, four sums a chunk.  (Launches in a row, weights from HBM; from L2 as much.  A launch by itself behind a
// flush of L2 takes 25 us for 64 rows.)
//
// Every wait is bounded; where one runs out the outputs of the cluster are NaN.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

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

__device__ __forceinline__ void cp_async_4(uint32_t dst, const float *src)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

// copies and instructions in flight get this long at least before their memory is given up
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

// Values of a word's codes 2 b and 2 b + 1 (byte b) as a pair of 16-bit numbers, in that order.  The fields
// c + 8 stay where the byte has them, in the low half at bit 0 and in the high half at bit 4: as denormal
// numbers, which two different powers of two make (c + 8) 2^-6 (bf16) or 2^-9 (fp16) of, exactly, in the
// fused operation that takes 8 or 7.5 of them off.
template <int XT> __device__ __forceinline__ uint32_t byte_values(uint32_t w, int b, uint32_t less)
{
    const uint32_t y = __byte_perm(w, w, 0x1111 * b);
    uint32_t v;                       // (y & mask) ^ sign bits
    asm("lop3.b32 %0, %1, %2, %3, 0x6a;" : "=r"(v) : "r"(y), "r"(0x00F0000Fu), "r"(0x00800008u));
    if (XT == DSQ_BF16) {
        const uint32_t scale = 0x7D007F00u;                       // 2^123, 2^127
        const __nv_bfloat162 r = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&v),
                                         *reinterpret_cast<const __nv_bfloat162 *>(&scale),
                                         *reinterpret_cast<const __nv_bfloat162 *>(&less));
        return *reinterpret_cast<const uint32_t *>(&r);
    }
    const uint32_t scale = 0x68007800u;                           // 2^11, 2^15
    const __half2 r = __hfma2(*reinterpret_cast<const __half2 *>(&v), *reinterpret_cast<const __half2 *>(&scale),
                              *reinterpret_cast<const __half2 *>(&less));
    return *reinterpret_cast<const uint32_t *>(&r);
}
// -7.5 or -8 units, twice, and what the sums are then multiples of (int8 values are 8 (2 c + 1) or 16 c)
template <int XT> __device__ __forceinline__ uint32_t byte_less(int odd)
{
    return XT == DSQ_BF16 ? (odd ? 0xBDF0BDF0u : 0xBE00BE00u) : (odd ? 0xA380A380u : 0xA400A400u);
}
template <int XT> __device__ __forceinline__ float byte_unit(int odd)
{
    return XT == DSQ_I8 ? (odd ? 0.125f : 0.0625f) : XT == DSQ_BF16 ? (odd ? 128.f : 64.f) : (odd ? 1024.f : 512.f);
}

// MC: columns of D that are read (rows of X); GP: pieces of 32 codes of a sum; TEAMS: of four warps that
// make values; COLS, TURNS: teams that take the sums, by columns and by chunks in turn
template <int XT, int MC, int GP, int TEAMS, int COLS, int TURNS, int STAGES> struct Layout {
    static constexpr bool INT = XT == DSQ_I8;
    static constexpr int NC = MC < 16 ? 16 : MC;                  // columns of an instruction
    static constexpr int FLUSHES = 4 / GP;                        // sums of a chunk
    static constexpr int AC = INT ? 32 : 64;                      // tensor-memory columns of a chunk's values
    static constexpr int VALUES = 6, ROOM = (512 - VALUES * AC) / NC;         // places for values
    static constexpr int SLOTS = FLUSHES == 1 ? (ROOM >= 6 ? 6 : ROOM >= 4 ? 4 : 2) : ROOM >= 8 ? 8 : ROOM >= 4 ? 4 : 2;
    static constexpr int A_COL = SLOTS * NC;                      // (places for sums)
    static constexpr int TAKES = COLS * TURNS, AHEAD = 8 / TURNS; // a team's chunks whose scales are on their way
    static constexpr int XBOX = NC * 128, XBOXES = INT ? 2 : 4;   // 128 bytes of K of the rows; of two chunks
    static constexpr int WBOX = 128 * 128, STAGE = WBOX + XBOXES * XBOX;
    static constexpr int RING_AT = 1024, S_AT = RING_AT + STAGES * STAGE, S_STAGE = FLUSHES * 512;
    static constexpr int BYTES = S_AT + TAKES * AHEAD * S_STAGE + 1024;      // (its start is aligned to 1024)
    // Warps that issue, chunks in turn: two where a place's sums are always the same one's.  (A warp knows a
    // place's use before the last to be over only from its own wait for it; else a phase's parity could be
    // an older one's.)
    static constexpr int ISSUERS = SLOTS % (2 * FLUSHES) == 0 ? 2 : 1;
    static constexpr int WORKERS = (TEAMS + TAKES) * 128, THREADS = WORKERS + 96;
    // barriers: a stage is full and empty, values made and read, sums ready and place free, all is done
    static constexpr int FULL = 16, EMPTY = FULL + 8 * STAGES, MADE = EMPTY + 8 * STAGES, READ = MADE + 8 * VALUES;
    static constexpr int READY = READ + 8 * VALUES, FREE = READY + 8 * SLOTS, DONE = FREE + 8 * SLOTS;
    static_assert(DONE + 16 <= RING_AT, "barriers");
    static_assert(BYTES <= 227 * 1024 && BYTES > 116 * 1024, "one block an SM");
    static_assert(TURNS * MC * 512 <= STAGES * STAGE, "the totals take the ring's place");
    static_assert(TURNS == 1 || SLOTS % (2 * FLUSHES) == 0, "a place's sums are one team's");
    static_assert(VALUES % TEAMS == 0 && VALUES % 2 == 0, "a place's values are one team's, and one issuer's");
    // (a chunk whose place has been read tells its team that all stages up to its own were full)
    static_assert(VALUES <= 2 * STAGES && A_COL + VALUES * AC <= 512, "phases are waited for in order");
};

template <int XT, int MC, int GP, int TEAMS, int COLS, int TURNS, int STAGES>
__global__ void __launch_bounds__((TEAMS + COLS * TURNS) * 128 + 96, 1)
wgemm_group_tc_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
                      const DsqGroupGemm p, const int split, const unsigned long long wait_ns, const int skip)
{
    using L = Layout<XT, MC, GP, TEAMS, COLS, TURNS, STAGES>;
    constexpr bool INT = L::INT;
    constexpr int FLUSHES = L::FLUSHES, TAKES = L::TAKES, AHEAD = L::AHEAD, MCT = MC / COLS;
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
    const int every = (all + 1) >> 1, c0 = 2 * (int)((int64_t)every * rank / split);
    const int chunks = min(2 * (int)((int64_t)every * (rank + 1) / split), all) - c0, pairs = (chunks + 1) >> 1;
    const int last = (int)min((int64_t)127, p.N - 1 - n0);       // row of weights of this block

    if (warp == L::WORKERS / 32 && lane == 0) {
        tma_prefetch_desc(&map_w);
        tma_prefetch_desc(&map_x);
    }
    if (warp == 0) {
        tmem_alloc(smem, 512);
        tmem_relinquish();
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) {
            mbar_init(smem + L::FULL + 8 * i, 1);
            mbar_init(smem + L::EMPTY + 8 * i, 2);           // (its two chunks)
        }
        for (int i = 0; i < L::VALUES; ++i) {
            mbar_init(smem + L::MADE + 8 * i, 4);
            mbar_init(smem + L::READ + 8 * i, 1);
        }
        for (int i = 0; i < L::SLOTS; ++i) {
            mbar_init(smem + L::READY + 8 * i, 1);
            mbar_init(smem + L::FREE + 8 * i, 4 * COLS);
        }
        for (int i = 0; i < 2; ++i) mbar_init(smem + L::DONE + 8 * i, 1);
        mbar_init_fence();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = lds_32(smem);
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);    // this warp's 32 lanes
    const unsigned long long drain_ns = wait_ns > DRAIN_NS ? wait_ns : DRAIN_NS;
    bool ok = true;               // (a role whose wait ran out stops; the others' waits run out in turn)
    auto wait = [&](uint32_t bar, uint32_t parity) { ok = wait_warp(smem + bar, parity, wait_ns); return ok; };
    grid_dependency_wait();
    grid_launch_dependents();

    float total[MCT];                                            // (of the takers' threads)
#pragma unroll
    for (int i = 0; i < MCT; ++i) total[i] = 0.f;
    if (team < TEAMS) {
        // values of the chunks team, team + TEAMS, ...: a row of 128 codes a thread
        const uint32_t less = byte_less<XT>(p.odd), one = p.odd ? 0x08080808u : 0u;
        int v = team, stage = team >> 1;
        uint32_t v_phase = 1, s_phase = 0;
#pragma unroll 1
        for (int c = team; c < chunks; c += TEAMS) {
            // (in this order: that the place's last values have been read says that all stages before the
            // last STAGES are full, without which a phase's parity could be an older one's)
            if (c >= L::VALUES && !wait(L::READ + 8 * v, v_phase)) break;
            if (!wait(L::FULL + 8 * stage, s_phase)) break;
            tc_fence_after_sync();
            const uint32_t codes = smem + L::RING_AT + stage * L::STAGE + row * 128, to = lanes + L::A_COL + v * L::AC;
#pragma unroll
            for (int h = 0; h < L::AC / 32; ++h) {
                constexpr int P16 = INT ? 4 : 2;                  // 16-byte pieces of the row, 32 columns
                uint32_t a[32];
#pragma unroll
                for (int q = 0; q < P16; ++q) {
                    const uint4 w4 = lds_128(codes + (((4 * (c & 1) + P16 * h + q) ^ row) & 7) * 16);
                    const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if constexpr (INT) {
                            const uint32_t even = ((w[k] << 4) & 0xF0F0F0F0u) | one, odd = (w[k] & 0xF0F0F0F0u) | one;
                            a[8 * q + 2 * k] = __byte_perm(even, odd, 0x5140);
                            a[8 * q + 2 * k + 1] = __byte_perm(even, odd, 0x7362);
                        } else {
#pragma unroll
                            for (int e = 0; e < 4; ++e) a[16 * q + 4 * k + e] = byte_values<XT>(w[k], e, less);
                        }
                    }
                }
                tmem_st_32x32(to + 32 * h, a);
            }
            tmem_st_wait();
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem + L::MADE + 8 * v);
            v += TEAMS;
            if (v >= L::VALUES) {
                v -= L::VALUES;
                v_phase ^= 1;
            }
            stage = ((c + TEAMS) >> 1) % STAGES;
            s_phase = (((c + TEAMS) >> 1) / STAGES) & 1;
        }
    } else if (team < TEAMS + TAKES) {
        // A row's scales go through a ring of their own, each thread's copies for itself.  (A chunk ahead, in
        // registers, the wait for them was the kernel's time: 32 times 0.6 us.)
        const int turn = (team - TEAMS) / COLS;
        const uint32_t s_ring = smem + L::S_AT + (team - TEAMS) * (AHEAD * L::S_STAGE) + row * 4;
        const uint32_t from = lanes + (team - TEAMS) % COLS * MCT;
        const float *scales = p.scales + n0 + min(row, last);
        auto issue_s = [&](int i) {
            const int c = TURNS * i + turn;
            if (c < chunks) {
#pragma unroll
                for (int f = 0; f < FLUSHES; ++f) {
                    const int g = min(p.group_of((uint32_t)((c0 + c) * FLUSHES + f)), p.groups - 1);
                    cp_async_4(s_ring + (i % AHEAD) * L::S_STAGE + f * 512, scales + (int64_t)g * p.N);
                }
            }
            cp_async_commit();
        };
#pragma unroll 1
        for (int i = 0; i < AHEAD - 1; ++i) issue_s(i);
#pragma unroll 1
        for (int i = 0; TURNS * i + turn < chunks && ok; ++i) {
            cp_async_wait<AHEAD - 2>();
            float now[FLUSHES];
#pragma unroll
            for (int f = 0; f < FLUSHES; ++f)
                now[f] = __uint_as_float(lds_32(s_ring + (i % AHEAD) * L::S_STAGE + f * 512));
            issue_s(i + AHEAD - 1);
#pragma unroll
            for (int f = 0; f < FLUSHES; ++f) {
                const uint32_t use = (TURNS * i + turn) * FLUSHES + f, slot = use % L::SLOTS;
                wait(L::READY + 8 * slot, (use / L::SLOTS) & 1);
                if (!ok) break;
                tc_fence_after_sync();
                constexpr int STEP = MCT < 32 ? MCT : 32;
#pragma unroll
                for (int h = 0; h < MCT / STEP; ++h) {
                    uint32_t v[STEP];
                    ld_cols(from + slot * L::NC + h * STEP, v);
                    tmem_ld_wait();
                    if (h == MCT / STEP - 1) {                    // the place is free again
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
        }
        cp_async_wait<0>();
    } else if (warp == L::WORKERS / 32) {
        // copies: two chunks' codes of 128 rows, whole lines, and X's rows beside them
        int issued = 0;
        for (; issued < pairs; ++issued) {
            const int stage = issued % STAGES;
            if (issued >= STAGES && !wait(L::EMPTY + 8 * stage, ((issued / STAGES) & 1) ^ 1)) break;
            if (lane == 0 && issued != skip) {
                const uint32_t to = smem + L::RING_AT + stage * L::STAGE, bar = smem + L::FULL + 8 * stage;
                const int at = (c0 >> 1) + issued;
                mbar_arrive_expect_tx(bar, L::STAGE);
                tma_load_2d(to, &map_w, at * 128, (int)n0, bar);
#pragma unroll
                for (int b = 0; b < L::XBOXES; ++b)
                    tma_load_2d(to + L::WBOX + b * L::XBOX, &map_x, (at * L::XBOXES + b) * 128, m0, bar);
            }
            __syncwarp();
        }
        // no copy is under way when the block ends
        for (int i = max(0, issued - STAGES); i < issued; ++i)
            if (i != skip && !wait_warp(smem + L::FULL + 8 * (i % STAGES), (i / STAGES) & 1, drain_ns)) ok = false;
    } else {
        // Two warps issue, chunks in turn: what they do lies in every chunk's way (commits and waits 0.2 us a
        // chunk, instructions 0.013 us each), so places and most phases are constants of an unrolled loop.
        auto issue = [&](auto which) {
            constexpr int Q = decltype(which)::value, IS = L::ISSUERS, COUNT = L::AC / 8 / FLUSHES;
            constexpr int UNROLL = 12;
            static_assert(UNROLL % L::VALUES == 0 && UNROLL * FLUSHES % L::SLOTS == 0 && UNROLL % IS == 0, "constants");
            const uint32_t idesc = INT ? idesc_i8(L::NC, true, true) : (XT == DSQ_BF16 ? idesc_bf16(L::NC) : dsq_idesc_f16(L::NC));
            constexpr uint32_t X_HALF = (L::XBOXES / 2) * (L::XBOX >> 4);
            const uint64_t desc = smem_desc_sw128(smem + L::RING_AT + L::WBOX);
            const uint32_t hi = (uint32_t)(desc >> 32), x_first = (uint32_t)desc;
            uint32_t x_at = x_first;
            uint32_t full = L::FULL, s_phase = 0, odd = 0;        // odd: a round of the loop
#pragma unroll 1
            for (int base = 0; base + Q < chunks && ok; base += UNROLL, odd ^= 1) {
#pragma unroll
                for (int u = Q; u < UNROLL; u += IS) {
                    const int v = u % L::VALUES;
                    if (base + u >= chunks) break;
                    if (!wait(full, s_phase)) break;
                    if (!wait(L::MADE + 8 * v, (u / L::VALUES + odd * (UNROLL / L::VALUES)) & 1)) break;
#pragma unroll
                    for (int f = 0; f < FLUSHES; ++f) {
                        const int use = u * FLUSHES + f, slot = use % L::SLOTS;
                        if ((base > 0 || use >= L::SLOTS) &&
                            !wait(L::FREE + 8 * slot, (use / L::SLOTS + odd * (UNROLL * FLUSHES / L::SLOTS) + 1) & 1))
                            break;
                        tc_fence_after_sync();
                        constexpr int BLOCK = COUNT < 4 ? COUNT : 4;
#pragma unroll
                        for (int i = 0; i < COUNT; i += BLOCK) {
                            const int at = (f * COUNT + i) * 32;              // bytes into the chunk's rows
                            mma_ts_elect<INT, BLOCK>(tmem + slot * L::NC, tmem + L::A_COL + v * L::AC + (f * COUNT + i) * 8,
                                                     x_at + ((u & 1) * X_HALF + (((at >> 7) * L::XBOX + (at & 127)) >> 4)), hi,
                                                     idesc, i);
                        }
                        mma_commit_elect(smem + L::READY + 8 * slot);
                    }
                    if (!ok) break;
                    mma_commit_elect(smem + L::READ + 8 * v);
                    mma_commit_elect(smem + full + (L::EMPTY - L::FULL));
                    if (IS == 1 && !(u & 1)) continue;
                    x_at += L::STAGE >> 4;
                    full += 8;
                    if (full == L::FULL + 8 * STAGES) {
                        full = L::FULL;
                        x_at = x_first;
                        s_phase ^= 1;
                    }
                }
            }
            // no instruction is under way when tensor memory is given up
            mma_commit_elect(smem + L::DONE + 8 * Q);
            if (!wait_warp(smem + L::DONE + 8 * Q, 0, drain_ns)) ok = false;
        };
        if (warp == L::WORKERS / 32 + 1) issue(std::integral_constant<int, 0>());
        else if (L::ISSUERS == 2) issue(std::integral_constant<int, 1>());
    }
    tc_fence_before_sync();
    const int failed = __syncthreads_or(!ok);
    if (warp == 0) {
        tc_fence_after_sync();
        tmem_dealloc(lds_32(smem), 512);
    }
    // the totals of the teams and of the cluster's blocks, [row of X][row of weights], added in their order
    const uint32_t sums = smem + L::RING_AT;
    const float unit = byte_unit<XT>(p.odd), lost = __uint_as_float(0x7FC00000u);
    if (team >= TEAMS && team < TEAMS + TAKES) {
        const int at = (team - TEAMS) / COLS * MC + (team - TEAMS) % COLS * MCT;
#pragma unroll
        for (int i = 0; i < MCT; ++i) sts_32(sums + ((at + i) * 128 + row) * 4, __float_as_uint(failed ? lost : total[i]));
    }
    if (split > 1) cluster_sync_all();
    else __syncthreads();
    if (team < TEAMS + TAKES) {
        // (eight loads on their way together: rows', or blocks' where there are few rows)
        constexpr int ROWS = MC <= 16 ? 1 : 4, BLOCKS = MC <= 16 ? 8 : 2;
        const int step = (TEAMS + TAKES) * split;
        for (int m = rank + team * split; m < rows; m += ROWS * step) {
            float s[ROWS] = {};
            for (int r0 = 0; r0 < split; r0 += BLOCKS) {
                uint32_t v[BLOCKS][TURNS][ROWS];
#pragma unroll
                for (int r = 0; r < BLOCKS; ++r) {
                    const uint32_t there = (split > 1 ? map_to_cta(sums, min(r0 + r, split - 1)) : sums) + row * 4;
#pragma unroll
                    for (int j = 0; j < ROWS; ++j)
#pragma unroll
                        for (int t = 0; t < TURNS; ++t) {
                            const uint32_t at = there + (t * MC + m + j * step) * 512;
                            v[r][t][j] = m + j * step >= rows || r0 + r >= split ? 0u : split > 1 ? ld_cluster_32(at) : lds_32(at);
                        }
                }
#pragma unroll
                for (int r = 0; r < BLOCKS; ++r)
#pragma unroll
                    for (int j = 0; j < ROWS; ++j)
#pragma unroll
                        for (int t = 0; t < TURNS; ++t) s[j] += __uint_as_float(v[r][t][j]);
            }
#pragma unroll
            for (int j = 0; j < ROWS; ++j)
                if (m + j * step < rows && row <= last) p.store(m0 + m + j * step, n0 + row, s[j] * unit);
        }
    }
    if (split > 1) cluster_sync_all();    // nobody leaves while its sums are read
}

// rows of bytes, in boxes of 128 of them by box_rows, in the 128-byte swizzle; zeros behind the ends
int make_map(CUtensorMap *map, const void *base, uint64_t bytes, uint64_t rows, uint64_t pitch, int box_rows)
{
    const DsqEncodeTiledFn fn = dsq_encode_tiled_fn();
    if (!fn) return DSQ_ERR_CUDA;
    const cuuint64_t dims[2] = {bytes, rows}, strides[1] = {pitch};
    const cuuint32_t box[2] = {128, (cuuint32_t)box_rows}, step[2] = {1, 1};
    const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, step,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? DSQ_OK : DSQ_ERR_CUDA;
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
template <int XT, int MC, int GP, int TEAMS, int COLS, int TURNS, int STAGES>
int launch(const DsqGroupGemm &p, cudaStream_t s, double *est_us)
{
    using L = Layout<XT, MC, GP, TEAMS, COLS, TURNS, STAGES>;
    static std::atomic<unsigned long long> configured{0};
    static std::atomic<int> active[4];
    const auto kernel = wgemm_group_tc_kernel<XT, MC, GP, TEAMS, COLS, TURNS, STAGES>;
    const int st = dsq_allow_smem((const void *)kernel, L::BYTES, &configured);
    if (st) return st;
    const int64_t tiles = (p.N + 127) / 128, mt = (p.M + MC - 1) / MC;
    const int pairs = ((p.K + 127) / 128 + 1) / 2, sms = dsq_sm_count() > 0 ? dsq_sm_count() : 148;
    // Blocks along K.  us of a wave: its start and end, the cluster's sums, and a chunk's time by the sums it
    // has; fitted to 216 sizes from 512 x 512 to 8192 x 8192 and 4 to 100 rows, within 12 % of nearly all.
    constexpr int AT = MC <= 8 ? 0 : MC <= 16 ? 1 : MC <= 32 ? 2 : 3, SUMS = GP == 4 ? 0 : GP == 2 ? 1 : 2;
    constexpr double START[] = {2.4, 3.4, 3.8, 5.4}, CLUSTER[] = {1.8, 1.2, 1.7, 0.8};
    constexpr double CHUNK[2][3][4] = {{{0.385, 0.39, 0.41, 0.435}, {0.45, 0.455, 0.48, 0.69}, {0.55, 0.56, 0.84, 0.965}},
                                       {{0.315, 0.32, 0.345, 0.385}, {0.38, 0.395, 0.43, 0.605}, {0.475, 0.505, 0.705, 0.925}}};
    int split = 1;
    double best = 1e30;
    for (int c = 1, k = 0; c <= 8 && c <= pairs; c *= 2, ++k) {
        const int64_t at_once = c == 1 ? sms : active_clusters(kernel, c, L::THREADS, L::BYTES, &active[k]);
        const double waves = (double)((tiles * mt + at_once - 1) / at_once);
        const double t = waves * (START[AT] + CHUNK[L::INT][SUMS][AT] * 2 * ((pairs + c - 1) / c)) + (c > 1 ? CLUSTER[AT] : 0.0);
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
    CUtensorMap map_w, map_x;
    const int row_bytes = p.K * (L::INT ? 1 : 2);
    int st2 = make_map(&map_w, p.W, (uint64_t)p.pitch, (uint64_t)p.N, (uint64_t)p.pitch, 128);
    if (!st2) st2 = make_map(&map_x, p.X, (uint64_t)row_bytes, (uint64_t)p.M, (uint64_t)row_bytes, L::NC);
    if (st2) return st2;
    const DsqLaunchHooks h = dsq_launch_hooks();
    return dsq_launch(kernel, dim3((unsigned)(tiles * split), (unsigned)mt), dim3(L::THREADS), (size_t)L::BYTES, s,
                      h.pdl, split, map_w, map_x, p, split, h.wait_ns, h.skip_b_round);
}

// Three teams make values (8192 x 8192, us, two and three: 16 rows 17.0 and 16.4, 64 rows 20.5 and 20.2).  Two take sums in
// turn where places allow (groups of 32, 8 rows, one and two: 24.8 and 20.6); with 64 rows two share the columns
// instead, for the registers.
template <int XT, int GP> int pick(const DsqGroupGemm &p, cudaStream_t s, double *est_us)
{
    constexpr bool INT = XT == DSQ_I8;
    if (p.M <= 8) return launch<XT, 8, GP, 3, 1, 2, 8>(p, s, est_us);
    if (p.M <= 16) return launch<XT, 16, GP, 3, 1, 2, 8>(p, s, est_us);
    if (p.M <= 32) return launch<XT, 32, GP, 3, 1, GP == 1 && !INT ? 1 : 2, INT ? 8 : 4>(p, s, est_us);
    return launch<XT, 64, GP, 3, 2, 1, 4>(p, s, est_us);
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
