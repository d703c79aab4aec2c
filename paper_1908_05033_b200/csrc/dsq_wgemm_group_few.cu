// Products of one or a few rows with 4-bit weights that have a scale per group: every operand
// an integer of 8 bits (dsq_wgemm_group.cu states the product).
//
// With a row or two the codes pass through the SM once, and what a code costs in instructions
// bounds the kernel: as bf16 a word of eight codes takes twelve to unpack and four instructions'
// worth of mma.sync, as int8 three and one (the field in the upper half of a byte is 16 c as it
// stands, with bit 3 set 8 (2 c + 1)).  So rows in 16 bits are made integers too: of each 256
// elements of a row the largest magnitude's exponent gives a power of two that takes it below
// 2^30, the element is cut into four signed digits of 8 bits, and the digits are four
// rows of the instruction, whose other rows would be empty anyway.  An element of bf16 (fp16) is
// whole down to 2^-22 (2^-19) of the largest of its 256.  Where one is not, what the digits leave
// of it goes through the same again, on a grid of its own, until nothing is left: whatever stands
// beside an element, its product is exact, as in the kernels for more rows.  (Of chunks of normal elements with
// one 12 times as large 3 in ten thousand take a second time, with one of 2^10 3 in a hundred, of 2^14 41: 8192 x 8192 with
// such an element in every chunk 10.7, 11.3 and 13.9 us.)
// Sums of up to 128 codes are exact in int32; they enter the totals times the group's scale and the
// power of two in binary32.
//
//   * A warp takes the chunks of 256 codes of 8 NT columns in turn with the others of its
//     block, through a ring of stages of its own in shared memory (cp.async, no barrier between
//     warps): the chunk's codes, the scales of its groups and its elements of X.  Lane (n = lane / 4,
//     j = lane & 3) has word j of each of a chunk's eight pieces of 32 codes of column n.
//   * The warps' totals, and then the digits' ones, are added in a fixed order.
//
// One row of bf16, us (at the copy's rate the codes and scales take): 4096 x 4096 4.8 (1.4), 8192 x 8192
// 10.6 (5.5), 16384 x 8192 19.4 (11.1), launches in a row with the weights from HBM; from L2 0.4 to 1.2
// less, a launch by itself behind a flush of L2 22.5 at 16384 x 8192.  Two rows of 8192 x 8192 12.2.  (With three
// digits, which lost what lies 2^-22 below a chunk's largest, one row 4.7, 10.1 and 18.6.)  Bound: latency of 16
// warps an SM (issue slots 54 %, memory 39 %).  Registers and shared memory allow two blocks; a third stage
// leaves room for one, and fewer or more columns or warps were slower (three digits, 8192 x 8192: three stages
// with one block 12.3, two or eight words of columns 11.8 and 11.7, 16 warps 13.0).
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

// the same on sums of zero
__device__ __forceinline__ void mma_i8_first(int (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
        "{%8, %9}, {%10, %10, %10, %10};"
        : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "r"(0));
}
__device__ __forceinline__ void sts_64(uint32_t at, uint32_t a, uint32_t b)
{
    asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(at), "r"(a), "r"(b) : "memory");
}
__device__ __forceinline__ void cp_async_4(uint32_t dst, const void *src, uint32_t src_bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(src_bytes) : "memory");
}

// A row of digits, 256 bytes in shared memory: where byte `at` of row n lies, so that rows meet no bank twice in
// 16-byte reads (GP = 4) or in 8-byte ones.
template <int GP> __device__ __forceinline__ uint32_t digit_at(int n, int at)
{
    return n * 256 + (GP == 4 ? at ^ ((n & 1) << 4) : at ^ ((n & 3) << 5));
}

// The grid of elements whose largest magnitude has the exponent field e: step = 2^(e - 156), 2^-149 at least (nothing of
// 16 bits lies below it); one over it as up1 up2, up2 other than 1 where binary32 does not hold it.
struct Grid { float up1, up2, step; };
__device__ __forceinline__ Grid grid_of(uint32_t e)
{
    const int k = 156 - (int)max(e, 7u), k1 = min(k, 126);
    Grid g;
    g.up1 = __uint_as_float((uint32_t)(127 + k1) << 23);
    g.up2 = __uint_as_float((uint32_t)(127 + k - k1) << 23);
    g.step = __uint_as_float(k <= 126 ? (uint32_t)(127 - k) << 23 : 1u << (149 - k));
    return g;
}
constexpr float MAGIC = 12582912.f;                           // 1.5 2^23

// Rows of X, one of them or both.  (One alone, known when compiling, is ordered worse by the compiler:
// 8192 x 8192 11.3 us against 10.1.)
constexpr int ROWS = 2, DIGITS = 4;

// GP: pieces of 32 codes that no group's end cuts
template <int XT, int NT, int GP, int WARPS, int STAGES> struct Few {
    static constexpr int FLUSHES = 8 / GP;
    static constexpr int W_BYTES = NT * 1024, S_BYTES = FLUSHES * NT * 32;
    static constexpr int STAGE = W_BYTES + S_BYTES + ROWS * 512;
    static constexpr int WARP_BYTES = STAGES * STAGE + ROWS * DIGITS * 256;
    static constexpr int SUMS = WARPS * NT * 64 * 4;
    static constexpr int BYTES = WARPS * WARP_BYTES > SUMS ? WARPS * WARP_BYTES : SUMS;
    static_assert(ROWS * DIGITS <= 8 && WARP_BYTES % 16 == 0 && BYTES <= 227 * 1024, "shared memory");
};

template <int XT, int NT, int GP, int WARPS, int STAGES>
__global__ void __launch_bounds__(WARPS * 32)
wgemm_group_few_kernel(const DsqGroupGemm p)
{
    using L = Few<XT, NT, GP, WARPS, STAGES>;
    constexpr int FLUSHES = L::FLUSHES;
    extern __shared__ __align__(128) uint8_t smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n = lane >> 2, j = lane & 3;
    const int64_t n0 = (int64_t)blockIdx.x * (8 * NT);
    const int m0 = blockIdx.y * ROWS, rows = min(p.M - m0, ROWS);
    const int chunks = (p.K + 255) >> 8;
    const int turns = warp < chunks ? (chunks - warp - 1) / WARPS + 1 : 0;
    const uint32_t ring = smem_u32(smem) + (uint32_t)(warp * L::WARP_BYTES), digits = ring + STAGES * L::STAGE;
    const int cols = (int)min((int64_t)8 * NT, p.N - n0);             // of this block

    // Codes: 16-byte piece j of each 64 bytes of column n of each eight, where the reads of a piece's
    // words meet no bank twice.  (Columns behind the last are the last: their sums are not used.)
    const uint8_t *src = p.W + n0 * p.pitch;
    int col_at[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) col_at[t] = min(8 * t + n, cols - 1) * p.pitch;
    const uint32_t w_to = n * 64 + ((j ^ (n >> 1)) & 3) * 16;
    // X: elements 8 lane .. 8 lane + 7 of the chunk
    const uint8_t *xs = p.X + (int64_t)m0 * p.K * 2 + lane * 16;
    const int64_t x_step = (int64_t)p.K * 2;
    const bool fours = (p.N & 3) == 0;                               // scales of four columns are aligned
    uint32_t stage_to = ring;
    int c_to = warp;                                                 // chunk that is copied next
    auto issue = [&]() {
        const int k_at = c_to * 128 + 16 * j;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const bool in = k_at + 64 * h < p.pitch;
            const uint8_t *s = src + (in ? k_at + 64 * h : 0);
            const uint32_t bytes = in ? 16u : 0u;
#pragma unroll
            for (int t = 0; t < NT; ++t) cp_async_16(stage_to + w_to + (2 * t + h) * 512, s + col_at[t], bytes);
        }
        const uint32_t s_to = stage_to + L::W_BYTES;
        if (fours) {
#pragma unroll
            for (int e = lane; e < FLUSHES * NT * 2; e += 32) {
                const int f = e / (NT * 2), c = e % (NT * 2) * 4, g = p.group_of((uint32_t)(c_to * FLUSHES + f));
                const bool in = g < p.groups && c < cols;
                cp_async_16(s_to + e * 16, in ? p.scales + (int64_t)g * p.N + n0 + c : p.scales, in ? 16u : 0u);
            }
        } else {
#pragma unroll
            for (int e = lane; e < FLUSHES * NT * 8; e += 32) {
                const int f = e / (NT * 8), c = e % (NT * 8), g = p.group_of((uint32_t)(c_to * FLUSHES + f));
                const bool in = g < p.groups && c < cols;
                cp_async_4(s_to + e * 4, in ? p.scales + (int64_t)g * p.N + n0 + c : p.scales, in ? 4u : 0u);
            }
        }
        const bool x_in = c_to * 256 + 8 * lane < p.K;
        const uint8_t *xm = xs + (x_in ? c_to * 512 : 0);
#pragma unroll
        for (int m = 0; m < ROWS; ++m) {
            const bool in = x_in && m < rows;
            cp_async_16(s_to + L::S_BYTES + m * 512 + lane * 16, in ? xm + m * x_step : p.X, in ? 16u : 0u);
        }
        c_to += WARPS;
        stage_to = stage_to == ring + (STAGES - 1) * L::STAGE ? ring : stage_to + L::STAGE;
    };

    grid_dependency_wait();
    grid_launch_dependents();
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) {
        if (s < turns) issue();
        cp_async_commit();
    }

    float total[NT][2];           // of the lower eight rows; the others are empty
#pragma unroll
    for (int t = 0; t < NT; ++t) total[t][0] = total[t][1] = 0.f;
    const uint32_t one = p.odd ? 0x08080808u : 0u;
    const uint32_t w_at = GP == 4 ? w_to : n * 64 + 4 * j;
    uint32_t at = ring;

#pragma unroll 1
    for (int i = 0; i < turns; ++i) {
        cp_async_wait<STAGES - 2>();
        __syncwarp();             // the stage is here; the last one, and the digits, have been read
        if (i + STAGES - 1 < turns) issue();
        cp_async_commit();
        const uint32_t s_at = at + L::W_BYTES, x_at = s_at + L::S_BYTES + lane * 16;
        int more = 0;             // elements are not whole on the grid of this turn of theirs
#pragma unroll 1
        for (int pass = 0; pass == 0 || more; ++pass) {
            if (pass > 0) __syncwarp();                           // the digits have been read
            // digits of X, in the order in which codes come out of their words; what this lane's row of sums is a
            // multiple of
            float up = 1.f;
            more = 0;
#pragma unroll
            for (int m = 0; m < ROWS; ++m) {
                if (m >= rows) break;
                const uint4 x = lds_128(x_at + m * 512);
                constexpr uint32_t ABS = 0x7FFF7FFFu, INF = XT == DSQ_BF16 ? 0x7F80u : 0x7C00u;
                const uint32_t t2 = __vmaxu2(__vmaxu2(x.x & ABS, x.y & ABS), __vmaxu2(x.z & ABS, x.w & ABS));
                const uint32_t top = __reduce_max_sync(~0u, max(t2 & 0xFFFFu, t2 >> 16));
                float f[8];
                DsqRaw8<__half> raw;
                raw.v[0] = x;
                uint32_t e;                      // the largest's exponent, as binary32 keeps it
                if (XT == DSQ_BF16) {
                    dsq_unpack8(reinterpret_cast<const DsqRaw8<__nv_bfloat16> &>(raw), f);
                    e = top >> 7;
                } else {
                    dsq_unpack8(raw, f);
                    e = __float_as_uint(__half2float(__ushort_as_half((unsigned short)top))) >> 23;
                }
                Grid g = grid_of(e);
#pragma unroll 1
                for (int p0 = 0; p0 < pass; ++p0) {              // what the digits before left
                    uint32_t most = 0;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        f[k] = __fmaf_rn(-rintf(f[k] * g.up2 * g.up1), g.step, f[k]);
                        most = max(most, __float_as_uint(f[k]) & 0x7FFFFFFFu);
                    }
                    g = grid_of(__reduce_max_sync(~0u, most) >> 23);
                }
                const bool bad = top >= INF;     // (rows with an infinity or a NaN: NaN)
                // whether all of an element is on the grid (numbers of eleven bits: those above 2^11 steps are whole, and
                // their sum with MAGIC is exact)
                if (g.step > 65536.f) {          // (of the smallest numbers times up1 nothing is left)
                    float lost = 0.f;
#pragma unroll
                    for (int k = 0; k < 8; ++k) lost = fmaxf(lost, fabsf(__fmaf_rn(-rintf(f[k] * g.up1), g.step, f[k])));
                    if (lost > 0.f && !bad) more = 1;
                } else if (g.up2 != 1.f) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) f[k] *= g.up2;
                }
                uint32_t v[8], dig[DIGITS][2];
#pragma unroll
                for (int k = 0; k < 8; ++k) {    // the integer plus 0x808080: its low bytes are digits plus 128
                    const float u = f[k] * g.up1;
                    if (__fsub_rn(__fadd_rn(u, MAGIC), MAGIC) != u && !bad) more = 1;
                    v[k] = (uint32_t)__float2int_rn(u) + 0x808080u;
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t a = __byte_perm(v[h], v[h + 2], 0x5140), b = __byte_perm(v[h + 4], v[h + 6], 0x5140);
                    const uint32_t c = __byte_perm(v[h], v[h + 2], 0x7362), d = __byte_perm(v[h + 4], v[h + 6], 0x7362);
                    dig[0][h] = __byte_perm(c, d, 0x7632);
                    dig[1][h] = __byte_perm(c, d, 0x5410) ^ 0x80808080u;
                    dig[2][h] = __byte_perm(a, b, 0x7632) ^ 0x80808080u;
                    dig[3][h] = __byte_perm(a, b, 0x5410) ^ 0x80808080u;
                }
#pragma unroll
                for (int k = 0; k < DIGITS; ++k) sts_64(digits + digit_at<GP>(DIGITS * m + k, 8 * lane), dig[k][0], dig[k][1]);
                if (n / DIGITS == m) up = bad ? __uint_as_float(0x7FC00000u) : g.step;
            }
            more = __any_sync(~0u, more);
            __syncwarp();
            // Operands: with groups of whole 128s lane j takes the four words of a 16-byte piece one after the
            // other (its codes 32 j .. 32 j + 31), else word j of each piece.
            uint32_t w[2][NT][4], a[8][2];
            const bool has_row = n < DIGITS * rows;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const uint32_t from = at + w_at + (2 * t + h) * 512;
                    if (GP == 4) {
                        const uint4 v = lds_128(from);
                        w[h][t][0] = v.x; w[h][t][1] = v.y; w[h][t][2] = v.z; w[h][t][3] = v.w;
                    } else {
#pragma unroll
                        for (int q = 0; q < 4; ++q) w[h][t][q] = lds_32(from + ((q ^ (n >> 1)) & 3) * 16);
                    }
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) a[4 * h + q][0] = a[4 * h + q][1] = 0u;
                if (GP == 4) {
#pragma unroll
                    for (int q = 0; q < 4; q += 2)
                        if (has_row) {
                            const uint4 v = lds_128(digits + digit_at<GP>(n, 128 * h + 32 * j + 8 * q));
                            a[4 * h + q][0] = v.x; a[4 * h + q][1] = v.y;
                            a[4 * h + q + 1][0] = v.z; a[4 * h + q + 1][1] = v.w;
                        }
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (has_row) {
                            const uint2 v = lds_64(digits + digit_at<GP>(n, 128 * h + 32 * q + 8 * j));
                            a[4 * h + q][0] = v.x; a[4 * h + q][1] = v.y;
                        }
                }
            }
            int acc[NT][4];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const uint32_t x_rows[4] = {a[q][0], 0u, a[q][1], 0u};
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const uint32_t c = w[q >> 2][t][q & 3];
                    const uint32_t b0 = ((c << 4) & 0xF0F0F0F0u) | one, b1 = (c & 0xF0F0F0F0u) | one;
                    if (q % GP == 0) mma_i8_first(acc[t], x_rows, b0, b1);
                    else mma_i8(acc[t], x_rows, b0, b1);
                }
                if (q % GP == GP - 1) {
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const uint2 sv = lds_64(s_at + ((q / GP) * NT * 8 + 8 * t + 2 * j) * 4);
                        total[t][0] = __fmaf_rn((float)acc[t][0] * up, __uint_as_float(sv.x), total[t][0]);
                        total[t][1] = __fmaf_rn((float)acc[t][1] * up, __uint_as_float(sv.y), total[t][1]);
                    }
                }
            }
        }
        at = at == ring + (STAGES - 1) * L::STAGE ? ring : at + L::STAGE;
    }
    cp_async_wait<0>();
    __syncthreads();
    float *sums = reinterpret_cast<float *>(smem);          // [WARPS][rows of digits][8 NT columns]
    constexpr int C = 8 * NT;
#pragma unroll
    for (int t = 0; t < NT; ++t)
        *reinterpret_cast<float2 *>(sums + (warp * 8 + n) * C + 8 * t + 2 * j) = make_float2(total[t][0], total[t][1]);
    __syncthreads();
    const float unit = dsq_value_unit<DSQ_I8>(p.odd);
    for (int e = threadIdx.x; e < rows * C; e += WARPS * 32) {
        const int m = e / C, col = e % C;
        if (col >= cols) continue;
        float d[DIGITS] = {};
#pragma unroll
        for (int k = 0; k < DIGITS; ++k)
#pragma unroll
            for (int w = 0; w < WARPS; ++w) d[k] += sums[(w * 8 + m * DIGITS + k) * C + col];
        p.store(m0 + m, n0 + col,
                __fmaf_rn(d[0], 16777216.f * unit, __fmaf_rn(d[1], 65536.f * unit, __fmaf_rn(d[2], 256.f * unit, d[3] * unit))));
    }
}

template <int XT, int NT, int GP, int WARPS, int STAGES> int launch(const DsqGroupGemm &p, cudaStream_t s)
{
    using L = Few<XT, NT, GP, WARPS, STAGES>;
    static std::atomic<unsigned long long> configured{0};
    const auto kernel = wgemm_group_few_kernel<XT, NT, GP, WARPS, STAGES>;
    const int st = dsq_allow_smem((const void *)kernel, L::BYTES, &configured);
    if (st) return st;
    const dim3 grid((unsigned)((p.N + 8 * NT - 1) / (8 * NT)), (unsigned)((p.M + ROWS - 1) / ROWS));
    return dsq_launch(kernel, grid, dim3(WARPS * 32), (size_t)L::BYTES, s, dsq_launch_hooks().pdl, 0, p);
}

template <int XT> int pick_group(DsqGroupGemm p, int64_t group, cudaStream_t s)
{
    const int gp = dsq_group_pieces(group);
    p.set_units(group, gp);
    return gp == 4 ? launch<XT, 4, 4, 8, 2>(p, s) : gp == 2 ? launch<XT, 4, 2, 8, 2>(p, s) : launch<XT, 4, 1, 8, 2>(p, s);
}

}  // namespace

int dsq_wgemm_group_few(const DsqGroupGemm &p, int x_type, int64_t group, cudaStream_t s)
{
    return x_type == DSQ_BF16 ? pick_group<DSQ_BF16>(p, group, s) : pick_group<DSQ_F16>(p, group, s);
}
