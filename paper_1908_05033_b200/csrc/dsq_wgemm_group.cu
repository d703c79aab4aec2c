// Products of few rows with 4-bit weights that have a scale per group (a decoder's linear
// layers while it serves):
//   Y[m][n] = row_scale[m] sum_g scale[g][n] sum_{k in g} X[m][k] v[n][k] + bias[n],
// v = 2 c + 1 or c, X bf16, fp16 (row_scale = 1) or int8.
//
// Three kernels: one or two rows of 16 bits as digits of 8 (dsq_wgemm_group_few.cu); this one, on
// mma.sync, where there is little work; tcgen05 where there is more (dsq_wgemm_group_tc.cu), by
// their estimated times.  (us of this one and of tcgen05: bf16, 8 rows, 4096 x 4096 5.9 and 7.9,
// 8192 x 8192 16.0 and 15.4; 64 rows 18 and 10.4, 64 and 20; int8, 8 rows, 8192 x 8192 9.8 and 12.9,
// 32 rows 21.5 and 15.0.)
//
// Here the codes are read once and used once: a warp takes them from global memory to tensor-core
// operands in registers, with one launch's latency and no hand-over between warps but at the
// end.  The sums of a group are kept apart (its products are exact in the tensor core's
// binary32, or int32, sums) and enter the total with the group's scale in binary32.  Bound: issue
// slots, of unpacking and of mma.sync whose 16 rows are M real ones.
//
//   * K is cut into chunks of 128 codes, a chunk into four pieces of 32 that never cross
//     a group.  Of a piece a lane (n = lane / 4, j = lane & 3) has word j of column n:
//     codes 8 j .. 8 j + 7, two k16 steps (one k32 step in int8); the order of K inside
//     a piece is free as long as both operands agree.
//   * bf16: the field of a code put into the upper mantissa bits of 1.0 is 1 + q / 16
//     (q = c + 8), and subtracting 1 + 7.5 / 16 (or 1.5) leaves (2 c + 1) / 32 (or c / 16)
//     exactly.  int8: the field in the upper half of a byte is 16 c as it stands, with bit 3
//     set 8 (2 c + 1).  The power of two goes into the scale.
//   * The warps of a block take the chunks of the same 8 NT columns in turn, each through a
//     ring of stages of its own in shared memory (cp.async; no barrier between warps), and
//     their totals are added in a fixed order at the end.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "dsq_groups.h"
#include "dsq_ptx.cuh"
#include "dsq_tc_host.h"
#include "dsq_types.cuh"
#include "dsq_wgemm_group.cuh"

using namespace dsq_ptx;

namespace {

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
__device__ __forceinline__ void mma_i8(int (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
        "{%8, %9}, {%0, %1, %2, %3};"
        : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void cp_async_4(uint32_t dst, const void *src, uint32_t src_bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(src_bytes) : "memory");
}
// rows: 8 (MT = 0: the lower half of an instruction's rows) or 16 MT
template <int MT> struct Rows { static constexpr int N = MT ? 16 * MT : 8, TILES = MT ? MT : 1; };
template <int XT> __host__ __device__ constexpr int x_bytes() { return XT == DSQ_I8 ? 128 : 256; }   // of a row's chunk
// bytes of a stage: codes of 8 NT columns, scales of 4 / GP groups, X of `rows` rows
template <int XT, int NT, int GP> __host__ __device__ constexpr int stage_bytes(int rows)
{
    return NT * 512 + (4 / GP) * NT * 32 + rows * x_bytes<XT>();
}

template <int XT, int MT, int NT, int GP, int WARPS, int STAGES>
__global__ void __launch_bounds__(WARPS * 32)
wgemm_group_kernel(const DsqGroupGemm p)
{
    constexpr int TILES = Rows<MT>::TILES, XB = x_bytes<XT>();
    constexpr bool INT = XT == DSQ_I8;
    extern __shared__ __align__(128) uint8_t smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n = lane >> 2, j = lane & 3;
    const int64_t n0 = (int64_t)blockIdx.x * (8 * NT);
    const int m0 = blockIdx.y * Rows<MT>::N;
    const int rows = min(p.M - m0, Rows<MT>::N);
    const int chunks = (p.K + 127) >> 7;
    const int turns = warp < chunks ? (chunks - warp - 1) / WARPS + 1 : 0;
    const int stage = stage_bytes<XT, NT, GP>(rows);
    const uint32_t ring = smem_u32(smem) + (uint32_t)(warp * STAGES * stage);
    const uint32_t base = dsq_value_base<XT>(p.odd);

    // the copies of this warp's i-th chunk into its stage
    auto issue_w = [&](int i) {
        if (i >= turns) return;
        const int c = warp + i * WARPS;
        const uint32_t at = ring + (uint32_t)(i % STAGES * stage);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            // 16-byte piece j of column n, where the reads of a piece's words meet no bank twice
            const int64_t col = n0 + 8 * t + n;
            const bool in = col < p.N && c * 64 + 16 * j < p.pitch;
            cp_async_16(at + t * 512 + n * 64 + ((j ^ (n >> 1)) & 3) * 16,
                        in ? p.W + col * p.pitch + c * 64 + 16 * j : p.W, in ? 16u : 0u);
        }
#pragma unroll
        for (int s = lane; s < (4 / GP) * NT * 8; s += 32) {
            const uint32_t unit = (uint32_t)(c * (4 / GP) + s / (8 * NT));
            const int g = p.group_of(unit);
            const int64_t col = n0 + s % (8 * NT);
            const bool in = g < p.groups && col < p.N;
            cp_async_4(at + NT * 512 + s * 4, in ? p.scales + (int64_t)g * p.N + col : p.scales, in ? 4u : 0u);
        }
    };
    auto issue_x = [&](int i) {
        if (i >= turns) return;
        const int c = warp + i * WARPS;
        const uint32_t at = ring + (uint32_t)(i % STAGES * stage + NT * 512 + (4 / GP) * NT * 32);
        constexpr int PIECES = XB / 16;
        for (int s = lane; s < rows * PIECES; s += 32) {
            const int row = s / PIECES, pc = s % PIECES;
            const bool in = (c * XB + 16 * pc) < p.K * (XB / 128);
            const int to = INT ? (((pc >> 1) ^ (row & 3)) << 1 | (pc & 1)) : pc ^ ((row & 1) << 2);
            cp_async_16(at + row * XB + to * 16,
                        in ? p.X + (int64_t)(m0 + row) * p.K * (XB / 128) + c * XB + 16 * pc : p.X, in ? 16u : 0u);
        }
    };

    grid_dependency_wait();
    grid_launch_dependents();
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) {
        issue_w(s);
        issue_x(s);
        cp_async_commit();
    }

    float total[TILES][NT][4];
#pragma unroll
    for (int m = 0; m < TILES; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) total[m][t][i] = 0.f;

#pragma unroll 1
    for (int i = 0; i < turns; ++i) {
        cp_async_wait<STAGES - 2>();
        __syncwarp();             // every lane's copies of this stage are here, and the last stage has been read
        issue_w(i + STAGES - 1);
        issue_x(i + STAGES - 1);
        cp_async_commit();
        const uint32_t at = ring + (uint32_t)(i % STAGES * stage);
        const uint32_t as = at + NT * 512, ax = as + (4 / GP) * NT * 32;
        typename std::conditional<INT, int, float>::type acc[TILES][NT][4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (q % GP == 0) {
#pragma unroll
                for (int m = 0; m < TILES; ++m)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[m][t][e] = 0;
            }
            // X of the piece: elements 8 j .. 8 j + 7 of rows n and n + 8 of each tile
            uint32_t a[TILES][2][4];
#pragma unroll
            for (int m = 0; m < TILES; ++m) {
                uint32_t x[2][4];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int row = 16 * m + 8 * h + n;
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[h][e] = 0u;
                    if (MT == 0 && h == 1) continue;
                    if (row < rows) {
                        if (INT) {
                            const uint2 v = lds_64(ax + row * XB + ((q ^ (row & 3)) << 5) + 8 * j);
                            x[h][0] = v.x; x[h][1] = v.y;
                        } else {
                            const uint4 v = lds_128(ax + row * XB + (((4 * q + j) ^ ((row & 1) << 2)) << 4));
                            x[h][0] = v.x; x[h][1] = v.y; x[h][2] = v.z; x[h][3] = v.w;
                        }
                    }
                }
                if (INT) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        a[m][0][h] = __byte_perm(x[h][0], x[h][1], 0x6420);
                        a[m][0][h + 2] = __byte_perm(x[h][0], x[h][1], 0x7531);
                    }
                } else {
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            // elements (2 s, 2 s + 4) and (2 s + 1, 2 s + 5)
                            a[m][s][h] = __byte_perm(x[h][s], x[h][s + 2], 0x5410);
                            a[m][s][h + 2] = __byte_perm(x[h][s], x[h][s + 2], 0x7632);
                        }
                }
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const uint32_t w = lds_32(at + t * 512 + n * 64 + ((q ^ (n >> 1)) & 3) * 16 + 4 * j);
                if constexpr (INT) {
                    const uint32_t one = p.odd ? 0x08080808u : 0u;
                    const uint32_t b0 = ((w << 4) & 0xF0F0F0F0u) | one, b1 = (w & 0xF0F0F0F0u) | one;
#pragma unroll
                    for (int m = 0; m < TILES; ++m) mma_i8(acc[m][t], a[m][0], b0, b1);
                } else {
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const uint32_t b0 = dsq_value_pair<XT>(w, 2 * s, base), b1 = dsq_value_pair<XT>(w, 2 * s + 1, base);
#pragma unroll
                        for (int m = 0; m < TILES; ++m) mma<XT>(acc[m][t], a[m][s], b0, b1);
                    }
                }
            }
            if (q % GP == GP - 1) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const uint2 sv = lds_64(as + (q / GP * NT * 8 + 8 * t + 2 * j) * 4);
                    const float s0 = __uint_as_float(sv.x), s1 = __uint_as_float(sv.y);
#pragma unroll
                    for (int m = 0; m < TILES; ++m) {
                        total[m][t][0] = __fmaf_rn((float)acc[m][t][0], s0, total[m][t][0]);
                        total[m][t][1] = __fmaf_rn((float)acc[m][t][1], s1, total[m][t][1]);
                        if (MT) {
                            total[m][t][2] = __fmaf_rn((float)acc[m][t][2], s0, total[m][t][2]);
                            total[m][t][3] = __fmaf_rn((float)acc[m][t][3], s1, total[m][t][3]);
                        }
                    }
                }
            }
        }
    }
    // the warps' totals, added in a fixed order
    cp_async_wait<0>();
    __syncthreads();
    float4 *part = reinterpret_cast<float4 *>(smem);        // [WARPS][TILES NT][32]
#pragma unroll
    for (int m = 0; m < TILES; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t)
            part[(warp * TILES * NT + m * NT + t) * 32 + lane] =
                make_float4(total[m][t][0], total[m][t][1], total[m][t][2], total[m][t][3]);
    __syncthreads();
    const float unit = dsq_value_unit<XT>(p.odd);
    const float *sums = reinterpret_cast<const float *>(smem);
    for (int e = threadIdx.x; e < TILES * NT * 128; e += WARPS * 32) {
        // element e of the tile in row-major order: 16 TILES rows, 8 NT columns
        const int col = e % (8 * NT), row = e / (8 * NT);
        if (row >= rows || n0 + col >= p.N) continue;
        const int tile = (row >> 4) * NT + (col >> 3);
        const int l = (row & 7) * 4 + ((col & 7) >> 1), k = 2 * ((row >> 3) & 1) + (col & 1);
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) s += sums[((w * TILES * NT + tile) * 32 + l) * 4 + k];
        p.store(m0 + row, n0 + col, s * unit);
    }
}

template <int XT, int MT, int NT, int GP, int WARPS, int STAGES> int launch(const DsqGroupGemm &p, cudaStream_t s)
{
    constexpr int ROWS = Rows<MT>::N;
    constexpr int most = WARPS * STAGES * stage_bytes<XT, NT, GP>(ROWS);
    constexpr int sums = WARPS * Rows<MT>::TILES * NT * 512;
    static_assert(most <= 227 * 1024 && sums <= most, "shared memory");
    static std::atomic<unsigned long long> configured{0};
    const auto kernel = wgemm_group_kernel<XT, MT, NT, GP, WARPS, STAGES>;
    const int st = dsq_allow_smem((const void *)kernel, most, &configured);
    if (st) return st;
    const int rows = p.M < ROWS ? p.M : ROWS;
    const int ring = WARPS * STAGES * stage_bytes<XT, NT, GP>(rows);
    const dim3 grid((unsigned)((p.N + 8 * NT - 1) / (8 * NT)), (unsigned)((p.M + ROWS - 1) / ROWS));
    return dsq_launch(kernel, grid, dim3(WARPS * 32), (size_t)(ring > sums ? ring : sums), s,
                      dsq_launch_hooks().pdl, 0, p);
}

template <int XT, int GP> int pick(const DsqGroupGemm &p, cudaStream_t s)
{
    if (p.M <= 8) return launch<XT, 0, 4, GP, 8, 3>(p, s);
    if (p.M <= 16) return launch<XT, 1, 4, GP, 8, 3>(p, s);
    if (p.M <= 32) return launch<XT, 2, 4, GP, 8, 2>(p, s);
    return launch<XT, 4, 4, GP, 4, 2>(p, s);
}

template <int XT> int pick_group(DsqGroupGemm p, int64_t group, cudaStream_t s)
{
    const int gp = dsq_group_pieces(group);
    p.set_units(group, gp);
    return gp == 4 ? pick<XT, 4>(p, s) : gp == 2 ? pick<XT, 2>(p, s) : pick<XT, 1>(p, s);
}

// Estimated time of these kernels: 1.6 us and the turns of a warp, times the blocks an SM has to run, those
// beyond its first at their share of it (8 rows: 2 and more are resident together) or in waves (one block
// an SM).  us of a turn, from 1024 x 8192 (one block an SM): 16-bit rows 9.5, 10.7, 15.3 and 32.1 us for 8, 16,
// 32 and 64 rows, int8 6.2, 7.6, 10.8 and 21.2.
double estimate_us(const DsqGroupGemm &p, bool i8)
{
    const int at = p.M <= 8 ? 0 : p.M <= 16 ? 1 : p.M <= 32 ? 2 : 3;
    static const double turn[2][4] = {{1.0, 1.15, 1.7, 1.9}, {0.58, 0.75, 1.15, 1.22}};
    const int warps = at == 3 ? 4 : 8, turns = ((p.K + 127) / 128 + warps - 1) / warps;
    const int sms = dsq_sm_count() > 0 ? dsq_sm_count() : 148;
    double load = (double)(((int64_t)p.N + 31) / 32 * ((p.M + 63) / 64)) / sms;
    const bool waves = i8 ? at == 2 : at != 0;
    if (load < 1.0) load = 1.0;
    if (waves) load = (double)(int64_t)(load + 0.999);
    return load * (1.6 + turns * turn[i8][at]);
}

}  // namespace

extern "C" int dsq_wgemm_group(const void *X, int x_type, const float *row_scale, const void *W_codes,
                               const float *scales, const float *bias, int64_t M, int64_t N, int64_t K,
                               int bits, int64_t group, float w_offset, int y_type, void *Y, void *stream)
{
    if (!X || !W_codes || !scales || !Y || (x_type == DSQ_I8 && !row_scale)) return DSQ_ERR_NULL;
    const int st = dsq_check_groups(N, K, bits, group);
    if (st) return st;
    if (M <= 0) return DSQ_ERR_SHAPE;
    if (!dsq_finite(w_offset)) return DSQ_ERR_RANGE;
    if ((x_type != DSQ_BF16 && x_type != DSQ_F16 && x_type != DSQ_I8) || !dsq_is_float_type(y_type) ||
        (w_offset != 0.0f && w_offset != 0.5f) || (x_type != DSQ_I8 && row_scale))
        return DSQ_ERR_UNSUPPORTED;
    const void *all[] = {X, row_scale, W_codes, scales, bias, Y};
    for (const void *a : all)
        if (!dsq_aligned16(a)) return DSQ_ERR_ALIGN;
    if (K % (x_type == DSQ_I8 ? 16 : 8) != 0) return DSQ_ERR_ALIGN;
    if (M > 65535 * 64) return DSQ_ERR_SIZE;
    // (a group longer than the row is the row.  Longer groups of 8-bit rows are refused as the interface has it: the
    // kernels take exact sums of 128 codes at most, which are far from int32's end.)
    const int64_t g = dsq_group_count(K, group) == 1 ? (K + 127) / 128 * 128 : group;
    if (x_type == DSQ_I8 && (g < K ? g : K) > (1 << 16)) return DSQ_ERR_OVERFLOW;
    DsqGroupGemm p;
    p.X = (const uint8_t *)X;
    p.W = (const uint8_t *)W_codes;
    p.scales = scales; p.bias = bias; p.row_scale = row_scale;
    p.Y = Y;
    p.N = N;
    p.M = (int)M; p.K = (int)K;
    p.pitch = (int)dsq_row_pitch(K, 4);
    p.groups = (int)dsq_group_count(K, g);
    p.units = p.units_inv = 0;
    p.odd = w_offset == 0.5f;
    p.y_type = y_type;
    cudaStream_t s = (cudaStream_t)stream;
    int form = dsq_launch_hooks().group_form;
    if (form == 3 && (x_type == DSQ_I8 || M > 2)) form = 1;
    if (form == 0 && x_type != DSQ_I8 && M <= 2) form = 3;
    if (form == 0) {
        double tc_us = 0.0;
        const int st2 = dsq_wgemm_group_tc(p, x_type, g, s, &tc_us);
        if (st2) return st2;
        form = tc_us < estimate_us(p, x_type == DSQ_I8) ? 2 : 1;
    }
    if (form == 3) return dsq_wgemm_group_few(p, x_type, g, s);
    if (form == 2) return dsq_wgemm_group_tc(p, x_type, g, s, nullptr);
    switch (x_type) {
    case DSQ_BF16: return pick_group<DSQ_BF16>(p, g, s);
    case DSQ_F16: return pick_group<DSQ_F16>(p, g, s);
    default: return pick_group<DSQ_I8>(p, g, s);
    }
}
