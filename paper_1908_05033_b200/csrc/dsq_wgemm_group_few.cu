// Products of one or a few rows with 4-bit weights that have a scale per group: every operand
// an integer of 8 bits (dsq_wgemm_group.cu states the product).
//
// With a row or two the codes pass through the SM once, and what a code costs in instructions
// bounds the kernel: as bf16 a word of eight codes takes twelve to unpack and four instructions'
// worth of mma.sync, as int8 three and one (the field in the upper half of a byte is 16 c as it
// stands, with bit 3 set 8 (2 c + 1)).  So rows in 16 bits are made integers too: of each 128
// elements of a row the largest magnitude's exponent gives a power of two that takes it below
// 2^22, the rounded element is cut into three signed digits of 8 bits, and the digits are three
// rows of the instruction, whose other rows would be empty anyway.  An element of
// bf16 (fp16) is exact down to 2^-14 (2^-11) of the largest of its 128, and below that off by at
// most 2^-22 of it.  Sums are exact in int32; they enter the totals times the group's scale and the
// power of two in binary32.
//
//   * A warp takes the chunks of 128 codes of 8 NT columns in turn with the others of its
//     block, through a ring of stages of its own in shared memory (cp.async, no barrier between
//     warps).  Lane (n = lane / 4, j = lane & 3) has word j of each of a chunk's four
//     pieces of 32 codes of column n.
//   * Rows of X and scales come a chunk ahead into registers.
//   * The warps' totals, and then the digits' ones, are added in a fixed order.
#include "dsq_groups.h"
#include "dsq_ptx.cuh"
#include "dsq_tc_host.h"
#include "dsq_types.cuh"
#include "dsq_wgemm_group.cuh"

using namespace dsq_ptx;

namespace {

__device__ __forceinline__ void mma_i8(int (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
        "{%8, %9}, {%0, %1, %2, %3};"
        : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

constexpr int ROW = 160;          // bytes of a row of digits in shared memory (rows meet no bank twice)

// HALF: at most 8 rows of digits (else 16); ROWS of X; GP: pieces of 32 codes that no group's end cuts
template <int XT, int ROWS, int NT, int GP, int WARPS, int STAGES> struct Few {
    static constexpr int DIGITS = XT == DSQ_I8 ? 1 : 3;
    static constexpr bool HALF = ROWS * DIGITS <= 8;
    static constexpr int W_BYTES = NT * 512;
    static constexpr int WARP_BYTES = STAGES * W_BYTES + ROWS * DIGITS * ROW;
    static constexpr int SUMS = WARPS * NT * (HALF ? 64 : 128) * 4;
    static constexpr int BYTES = WARPS * WARP_BYTES > SUMS ? WARPS * WARP_BYTES : SUMS;
    static_assert(ROWS * DIGITS <= 16 && WARP_BYTES % 16 == 0 && BYTES <= 227 * 1024, "shared memory");
};

template <int XT, int ROWS, int NT, int GP, int WARPS, int STAGES>
__global__ void __launch_bounds__(WARPS * 32)
wgemm_group_few_kernel(const DsqGroupGemm p)
{
    using L = Few<XT, ROWS, NT, GP, WARPS, STAGES>;
    constexpr int DIGITS = L::DIGITS, FLUSHES = 4 / GP, SLOTS = L::HALF ? 2 : 4;
    constexpr bool INT = XT == DSQ_I8;
    extern __shared__ __align__(128) uint8_t smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n = lane >> 2, j = lane & 3;
    const int64_t n0 = (int64_t)blockIdx.x * (8 * NT);
    const int m0 = blockIdx.y * ROWS, rows = min(p.M - m0, ROWS);
    const int chunks = (p.K + 127) >> 7;
    const int turns = warp < chunks ? (chunks - warp - 1) / WARPS + 1 : 0;
    const uint32_t ring = smem_u32(smem) + (uint32_t)(warp * L::WARP_BYTES), digits = ring + STAGES * L::W_BYTES;

    // codes: 16-byte piece j of column n of each eight, where the reads of a piece's words meet no
    // bank twice
    const uint8_t *src = p.W + (n0 + n) * p.pitch + warp * 64 + 16 * j;
    const uint32_t w_to = ring + n * 64 + ((j ^ (n >> 1)) & 3) * 16;
    const int64_t step = 8 * (int64_t)p.pitch;
    const int cols = (int)min((int64_t)8 * NT, p.N - n0);             // of this block
    int left = p.pitch - warp * 64 - 16 * j;                         // bytes of the rows from src on
    uint32_t w_stage = 0;
    auto issue = [&]() {
        const uint8_t *s = src;
#pragma unroll
        for (int t = 0; t < NT; ++t, s += step) {
            const bool in = left > 0 && 8 * t + n < cols;
            cp_async_16(w_to + w_stage + t * 512, in ? s : p.W, in ? 16u : 0u);
        }
        src += WARPS * 64;
        left -= WARPS * 64;
        w_stage = w_stage == (STAGES - 1) * L::W_BYTES ? 0u : w_stage + L::W_BYTES;
        cp_async_commit();
    };
    // X: elements 4 lane .. 4 lane + 3 of the chunk; scales of columns 8 t + 2 j and + 1
    uint2 x[ROWS];
    float2 sc[FLUSHES][NT];
    const uint8_t *xs = p.X + ((int64_t)m0 * p.K + warp * 128 + 4 * lane) * (INT ? 1 : 2);
    const bool pairs = (p.N & 1) == 0;
    auto load = [&](int i) {
        const int k = (warp + i * WARPS) * 128 + 4 * lane;
#pragma unroll
        for (int m = 0; m < ROWS; ++m) {
            x[m] = make_uint2(0u, 0u);
            if (i < turns && m < rows && k < p.K) {
                const uint8_t *at = xs + (int64_t)m * p.K * (INT ? 1 : 2);
                if (INT) x[m].x = __ldg(reinterpret_cast<const uint32_t *>(at));
                else x[m] = __ldg(reinterpret_cast<const uint2 *>(at));
            }
        }
        xs += WARPS * 128 * (INT ? 1 : 2);
#pragma unroll
        for (int f = 0; f < FLUSHES; ++f) {
            const int g = p.group_of((uint32_t)((warp + i * WARPS) * FLUSHES + f));
            const bool in = i < turns && g < p.groups;
            const float *s = p.scales + (int64_t)g * p.N + n0 + 2 * j;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int c = 8 * t + 2 * j;
                sc[f][t] = make_float2(0.f, 0.f);
                if (pairs) {
                    if (in && c < cols) sc[f][t] = __ldg(reinterpret_cast<const float2 *>(s + 8 * t));
                } else {
                    if (in && c < cols) sc[f][t].x = __ldg(s + 8 * t);
                    if (in && c + 1 < cols) sc[f][t].y = __ldg(s + 8 * t + 1);
                }
            }
        }
    };

    grid_dependency_wait();
    grid_launch_dependents();
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) issue();
    load(0);

    float total[NT][SLOTS];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < SLOTS; ++e) total[t][e] = 0.f;
    const uint32_t one = p.odd ? 0x08080808u : 0u;
    const uint32_t w_at = ring + n * 64 + 4 * j;
    uint32_t r_stage = 0;

#pragma unroll 1
    for (int i = 0; i < turns; ++i) {
        cp_async_wait<STAGES - 2>();
        __syncwarp();             // the stage is here; the last one, and the digits, have been read
        issue();
        // digits of X; what this lane's rows of sums (n, n + 8) are multiples of
        float up[2] = {1.f, 1.f};
        if (INT) {
#pragma unroll
            for (int m = 0; m < ROWS; ++m)
                if (m < rows) sts_32(digits + m * ROW + 4 * lane, x[m].x);
        } else {
#pragma unroll
            for (int m = 0; m < ROWS; ++m) {
                if (m >= rows) break;
                float f[4];
                if (XT == DSQ_BF16) {
                    f[0] = __uint_as_float(x[m].x << 16); f[1] = __uint_as_float(x[m].x & 0xFFFF0000u);
                    f[2] = __uint_as_float(x[m].y << 16); f[3] = __uint_as_float(x[m].y & 0xFFFF0000u);
                } else {
                    const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(&x[m].x));
                    const float2 b = __half22float2(*reinterpret_cast<const __half2 *>(&x[m].y));
                    f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y;
                }
                uint32_t top = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) top = max(top, __float_as_uint(f[e]) & 0x7FFFFFFFu);
                top = __reduce_max_sync(~0u, top);
                // 2^(21 - e) of the largest's exponent e, and its inverse (rows with an infinity or a NaN: NaN)
                const uint32_t e = max(top >> 23, 22u);
                const float scale = __uint_as_float((275u - e) << 23);
                const float inv = top >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : __uint_as_float((e - 21u) << 23);
                uint32_t v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k)      // the integer plus 0x8080: its low bytes are digits plus 128
                    v[k] = __float_as_uint(__fmaf_rn(f[k], scale, 12582912.f)) + (0x8080u - 0x4B400000u);
                const uint32_t a = __byte_perm(v[0], v[1], 0x5140), b = __byte_perm(v[2], v[3], 0x5140);
                const uint32_t to = digits + 3 * m * ROW + 4 * lane;
                sts_32(to, __byte_perm(__byte_perm(v[0], v[1], 0x0062), __byte_perm(v[2], v[3], 0x0062), 0x5410));
                sts_32(to + ROW, __byte_perm(a, b, 0x7632) ^ 0x80808080u);
                sts_32(to + 2 * ROW, __byte_perm(a, b, 0x5410) ^ 0x80808080u);
                if (n / 3 == m) up[0] = inv;
                if ((n + 8) / 3 == m) up[1] = inv;
            }
        }
        float2 now[FLUSHES][NT];
#pragma unroll
        for (int f = 0; f < FLUSHES; ++f)
#pragma unroll
            for (int t = 0; t < NT; ++t) now[f][t] = sc[f][t];
        load(i + 1);
        __syncwarp();
        int acc[NT][4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (q % GP == 0) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[t][e] = 0;
            }
            uint32_t a[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int h = 0; h < (L::HALF ? 1 : 2); ++h)
                if (n + 8 * h < rows * DIGITS) {
                    const uint2 v = lds_64(digits + (n + 8 * h) * ROW + q * 32 + 8 * j);
                    a[h] = __byte_perm(v.x, v.y, 0x6420);
                    a[h + 2] = __byte_perm(v.x, v.y, 0x7531);
                }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const uint32_t w = lds_32(w_at + r_stage + t * 512 + ((q ^ (n >> 1)) & 3) * 16);
                mma_i8(acc[t], a, ((w << 4) & 0xF0F0F0F0u) | one, (w & 0xF0F0F0F0u) | one);
            }
            if (q % GP == GP - 1) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const float2 s = now[q / GP][t];
#pragma unroll
                    for (int h = 0; h < SLOTS / 2; ++h) {
                        total[t][2 * h] = __fmaf_rn((float)acc[t][2 * h] * up[h], s.x, total[t][2 * h]);
                        total[t][2 * h + 1] = __fmaf_rn((float)acc[t][2 * h + 1] * up[h], s.y, total[t][2 * h + 1]);
                    }
                }
            }
        }
        r_stage = r_stage == (STAGES - 1) * L::W_BYTES ? 0u : r_stage + L::W_BYTES;
    }
    cp_async_wait<0>();
    __syncthreads();
    float *sums = reinterpret_cast<float *>(smem);          // [WARPS][rows of digits][8 NT columns]
    constexpr int R = L::HALF ? 8 : 16, C = 8 * NT;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int h = 0; h < SLOTS / 2; ++h)
            *reinterpret_cast<float2 *>(sums + (warp * R + n + 8 * h) * C + 8 * t + 2 * j) =
                make_float2(total[t][2 * h], total[t][2 * h + 1]);
    __syncthreads();
    const float unit = dsq_value_unit<DSQ_I8>(p.odd);
    for (int e = threadIdx.x; e < rows * C; e += WARPS * 32) {
        const int m = e / C, col = e % C;
        if (col >= cols) continue;
        float d[DIGITS];
#pragma unroll
        for (int k = 0; k < DIGITS; ++k) {
            d[k] = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) d[k] += sums[(w * R + m * DIGITS + k) * C + col];
        }
        float s = d[0];
        if (DIGITS == 3) s = __fmaf_rn(d[0], 65536.f, __fmaf_rn(d[1 % DIGITS], 256.f, d[2 % DIGITS]));
        p.store(m0 + m, n0 + col, s * unit);
    }
}

template <int XT, int ROWS, int NT, int GP, int WARPS, int STAGES> int launch(const DsqGroupGemm &p, cudaStream_t s)
{
    using L = Few<XT, ROWS, NT, GP, WARPS, STAGES>;
    static std::atomic<unsigned long long> configured{0};
    const auto kernel = wgemm_group_few_kernel<XT, ROWS, NT, GP, WARPS, STAGES>;
    const int st = dsq_allow_smem((const void *)kernel, L::BYTES, &configured);
    if (st) return st;
    const dim3 grid((unsigned)((p.N + 8 * NT - 1) / (8 * NT)), (unsigned)((p.M + ROWS - 1) / ROWS));
    return dsq_launch(kernel, grid, dim3(WARPS * 32), (size_t)L::BYTES, s, dsq_launch_hooks().pdl, 0, p);
}

template <int XT, int GP> int pick(const DsqGroupGemm &p, cudaStream_t s)
{
    if constexpr (XT == DSQ_I8) {
        if (p.M <= 8) return launch<XT, 8, 4, GP, 8, 4>(p, s);
        return launch<XT, 16, 4, GP, 8, 4>(p, s);
    } else {
        if (p.M == 1) return launch<XT, 1, 4, GP, 8, 4>(p, s);
        if (p.M == 2) return launch<XT, 2, 4, GP, 8, 4>(p, s);
        return launch<XT, 5, 4, GP, 8, 4>(p, s);
    }
}

template <int XT> int pick_group(DsqGroupGemm p, int64_t group, cudaStream_t s)
{
    const int gp = dsq_group_pieces(group);
    p.set_units(group, gp);
    return gp == 4 ? pick<XT, 4>(p, s) : gp == 2 ? pick<XT, 2>(p, s) : pick<XT, 1>(p, s);
}

}  // namespace

int dsq_wgemm_group_few(const DsqGroupGemm &p, int x_type, int64_t group, cudaStream_t s)
{
    switch (x_type) {
    case DSQ_BF16: return pick_group<DSQ_BF16>(p, group, s);
    case DSQ_F16: return pick_group<DSQ_F16>(p, group, s);
    default: return pick_group<DSQ_I8>(p, group, s);
    }
}
