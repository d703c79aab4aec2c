// A layer of experts for few tokens: the router's choice, and the chosen experts' gated layers on
// 4-bit weights with group scales (what stands in a decoder where dsq_wgemm_group would be twice).
//
//   mid = act(x W_gate^T) * (x W_up^T),   y_t = residual_t + sum_s weight_ts mid_ts W_out^T
//
// Bound by the bytes of the experts that anything goes to, read once: 128 bytes of codes that a warp reads
// may cost it some 18 instructions at 6 TB/s, and unpacking them to bf16 is 12 (dsq_wgemm_group.cu).
// So everything is 8-bit integers, as in dsq_wgemm_group_few.cu: a word of eight codes takes 3 instructions,
// a row of x or mid is four signed digits of 8 bits, on a grid of its own for each chunk of 128 elements
// (2^-30 of the largest's power of two), and four slots' digits are the 16 rows of an instruction.
//
//   * A slot is a token's s-th choice.  moe_prepare_kernel sorts the slots by expert (stable), cuts each
//     expert's into groups of up to four, and makes digits of x, as an instruction's rows want them.
//   * moe_in_kernel: a block has columns of a group's gate and the same ones of its other half; warps
//     split columns and K in chunks of 128 codes, each through a ring of stages of its own (cp.async,
//     no barrier between warps); their sums are added in a fixed order, and the activation makes
//     mid of them, in binary32.  moe_mid_kernel makes digits of it.
//   * moe_out_kernel: a cluster has columns of all tokens; the chunks of all groups, one behind the
//     other, are cut evenly among its warps, so that all have the same work however the tokens
//     are spread.  A warp adds a group's sums, times the tokens' weights, to rows of its own in shared memory;
//     at the end the warps' and the cluster's are added in a fixed order: no atomics, no partial results in
//     memory.  Its first codes are on their way while the kernels ahead still run.
//   * Sums of up to 128 codes are exact in int32; they enter the totals in binary32.  Digits leave of an
//     element what is below 2^-31 of the largest of its 128: for the codes' grid Delta (c + 1/2),
//     which has no 0, that is below the rounding of the sums.  The grid Delta c, whose 0 can make the largest
//     element vanish, and experts with more slots go on 16 bits (dsq_moe_wide.cu).
// One token of 2048 to 1024, eight of 64 experts (27 MB of codes and scales): 14 us, of which four launches in a row
// without work are 6 (14.4 against 13.6 where the first product's copies wait for the groups that the kernel ahead writes).  16
// tokens of 4096 to 1024, four of 64 (276 MB): 72 us, 3.8 TB/s; no unit is saturated (issue slots 56 % and 45 %, tensor pipe
// 27 % and 18 %, DRAM 52 % and 37 % in the two products): warps wait for digits from L1, for copies and for one another's
// instructions (275 a chunk of 2 KB: 97 for its copies, 187 to unpack and multiply).
#include "dsq_moe.cuh"

using namespace dsq_moe;

namespace {

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

__device__ __forceinline__ float value_of(uint32_t o)
{
    return __uint_as_float(o == 0u ? 0x7FC00000u : (int)o < 0 ? o & 0x7FFFFFFFu : ~o);
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
        const float value = value_of(last);
        if (s == 0) first = value;
        if (lane == s) {
            mine = value;
            my_id = last_at;
        }
    }
    // (where the largest is -infinity: less 0, which leaves sums of 0, or of a NaN below it)
    const float base = first == __uint_as_float(0xFF800000u) ? 0.f : first;
    float e = lane < p.k ? expf(mine - base) : 0.f, sum = e;
    if (!p.renormalise) {
        sum = 0.f;
        for (int i = lane; i < p.E; i += 32) sum += expf(row[i] - base);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    if (lane < p.k) {
        p.ids[t * p.k + lane] = my_id;
        p.weights[t * p.k + lane] = sum == 0.f ? 0.f : e / sum;
    }
}

// ---- preparation ---------------------------------------------------------------------------
// expert, n and the slots of a group of up to four
struct Members {
    int expert, n;
    uint2 slots;
    __device__ __forceinline__ int slot(int r) const
    {
        const uint32_t w = r & 2 ? slots.y : slots.x;
        return (int)(r & 1 ? w >> 16 : w & 0xFFFFu);
    }
    // of slots as bits, four at most
    __device__ __forceinline__ void set(uint32_t bits)
    {
        n = __popc(bits);
        uint32_t at[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            at[i] = bits ? (uint32_t)__ffs(bits) - 1 : 0u;
            bits &= bits - 1;
        }
        slots = make_uint2(at[0] | at[1] << 16, at[2] | at[3] << 16);
    }
};
__device__ __forceinline__ Members members_of(const Work &w, int i)
{
    const uint4 a = load_16(w.group + i), b = load_16(w.group[i].slot);
    return {(int)a.x, (int)a.y, make_uint2(b.x, b.y)};
}

// The four digits of a chunk of 128 elements, by a warp: f holds elements 4 lane .. 4 lane + 3.  512 bytes, as an
// instruction's rows want them: a lane of row n (and n + 8) has digits d = n & 1 (and d + 2) of a slot, and of each of its
// four words of codes 16 bytes: codes 0, 2, 4, 6 in digit d, in digit d + 2, codes 1, 3, 5, 7 in digit d, in digit d + 2; the
// words of lane j are 4 j .. 4 j + 3 where no group's end cuts the chunk (WHOLE), else j, j + 4, j + 8, j + 12.  The
// 16 bytes of word q of lane j and digit d lie at 128 q + 64 d + 16 j.  Returns what the highest digit (0) stands for.
template <bool WHOLE> __device__ __forceinline__ float make_digits(const float (&f)[4], uint8_t *to)
{
    const int lane = threadIdx.x & 31;
    float most = 0.f;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        most = fmaxf(most, fabsf(f[i]));
        bad = bad || !(fabsf(f[i]) <= 3.402823466e38f);
    }
    const uint32_t e = __reduce_max_sync(~0u, __float_as_uint(most) >> 23);
    // the lowest digit stands for 2^(e - 156), 2^-149 at least: the largest is below 2^30 of it
    const int up = 156 - (int)max(e, 7u), up1 = min(up, 126);
    const float a = __uint_as_float((uint32_t)(127 + up1) << 23), b = __uint_as_float((uint32_t)(127 + up - up1) << 23);
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = (uint32_t)__float2int_rn(f[i] * b * a) + 0x808080u;       // its lower bytes are digits plus 128
    }
    const int block = lane >> 1, half = lane & 1;
    const int j = WHOLE ? block >> 2 : block & 3, q = WHOLE ? block & 3 : block >> 2;
    uint8_t *at = to + q * 128 + j * 16 + half * 2;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        const uint32_t flip = d == 0 ? 0u : 0x8080u;
        const uint32_t sel = (3 - d) | (7 - d) << 4;
        uint8_t *digit = at + (d & 1) * 64 + (d >> 1) * 4;
        *reinterpret_cast<uint16_t *>(digit) = (uint16_t)(__byte_perm(v[0], v[2], sel) ^ flip);
        *reinterpret_cast<uint16_t *>(digit + 8) = (uint16_t)(__byte_perm(v[1], v[3], sel) ^ flip);
    }
    if (__any_sync(~0u, bad)) return __uint_as_float(0x7FC00000u);
    return __uint_as_float((uint32_t)(151 - up) << 23);       // 2^(24 - up)
}

constexpr int PREPARE_WARPS = 8;
// block 0: the slots; the others' warps a chunk of a token each
template <int XT, bool WHOLE> __global__ void __launch_bounds__(PREPARE_WARPS * 32) moe_prepare_kernel(const __grid_constant__ MoeParams p)
{
    __shared__ Sorting sorting;
    grid_dependency_wait();
    grid_launch_dependents();
    if (blockIdx.x == 0) {
        sort_slots(p, sorting);
        return;
    }
    const int i = (blockIdx.x - 1) * PREPARE_WARPS + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (i >= p.T * p.chunks_in) return;
    const int t = i / p.chunks_in, c = i - t * p.chunks_in, k = c * 128 + 4 * lane;
    float f[4] = {};
    if (k < p.H) {                    // (H is a multiple of 8)
        const uint2 v = *reinterpret_cast<const uint2 *>(p.X + ((int64_t)t * p.H + k) * 2);
        const uint32_t w[2] = {v.x, v.y};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (XT == DSQ_BF16) {
                f[2 * h] = __uint_as_float(w[h] << 16);
                f[2 * h + 1] = __uint_as_float(w[h] & 0xFFFF0000u);
            } else {
                const float2 u = __half22float2(*reinterpret_cast<const __half2 *>(&w[h]));
                f[2 * h] = u.x;
                f[2 * h + 1] = u.y;
            }
        }
    }
    const float step = make_digits<WHOLE>(f, p.w.x + (int64_t)i * 512);
    if (lane == 0) p.w.x_step[i] = step;
}

// mid's digits, a warp a chunk of a slot (of slots without an expert: of whatever lies there)
template <bool WHOLE> __global__ void __launch_bounds__(PREPARE_WARPS * 32) moe_mid_kernel(const __grid_constant__ MoeParams p)
{
    const int i = blockIdx.x * PREPARE_WARPS + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    grid_dependency_wait();
    grid_launch_dependents();
    if (i >= p.slots * p.chunks_out) return;
    const float4 v = *reinterpret_cast<const float4 *>(p.w.mid + (int64_t)i * 128 + 4 * lane);
    const float f[4] = {v.x, v.y, v.z, v.w};
    const float step = make_digits<WHOLE>(f, p.w.mid_rows + (int64_t)i * 512);
    if (lane == 0) p.w.mid_step[i] = step;
}

// ---- digits
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

// What a lane has of a chunk's rows, a tile being four slots: digits n & 1 and (n & 1) + 2 of slot n / 2, and the step.
template <int TILES> struct Digits {
    uint4 x[TILES][4];
    float step[TILES];
};
// where they are: slot r of a group has its chunks of digits and steps at `digits` and `steps`, from the lane's place on
template <int TILES> struct Sources {
    const uint8_t *digits[TILES];
    const float *steps[TILES];
    __device__ __forceinline__ void set(int m, const uint8_t *d, const float *s)
    {
        const int lane = threadIdx.x & 31;
        digits[m] = d ? d + (lane >> 2 & 1) * 64 + (lane & 3) * 16 : nullptr;
        steps[m] = s;
    }
    // (rows of no slot stay zeros)
    __device__ __forceinline__ void load(int chunk, Digits<TILES> &r) const
    {
#pragma unroll
        for (int m = 0; m < TILES; ++m)
            if (digits[m]) {
                const uint8_t *at = digits[m] + (int64_t)chunk * 512;
#pragma unroll
                for (int q = 0; q < 4; ++q) r.x[m][q] = load_16(at + 128 * q);
                r.step[m] = steps[m][chunk];
            }
    }
    // Brings a chunk into L1, a line a lane of eight (the loads behind would wait for L2 with every register taken).
    __device__ __forceinline__ void touch(int chunk) const
    {
#pragma unroll
        for (int m = 0; m < TILES; ++m)
            if (digits[m]) {
                const int lane = threadIdx.x & 31;
                uint32_t none;
                asm volatile("ld.global.u32 %0, [%1];" : "=r"(none) : "l"(digits[m] + (int64_t)chunk * 512 + (lane & 3) * 112));
            }
    }
};

// total += scale step (sum of digits times codes) of a chunk
template <int TILES, int NT, int GP>
__device__ __forceinline__ void multiply_digits(uint32_t at, const Digits<TILES> &r, DsqPair (&total)[TILES][NT][2])
{
    const int lane = threadIdx.x & 31, n = lane >> 2, j = lane & 3;
    const uint32_t as = at + Stage<NT, GP>::W_BYTES;
    constexpr uint32_t one = 0x08080808u;                     // codes 2 c + 1 (times 8)
    // (SIDE tiles of columns together: an instruction's sums are 20 clocks away from the next one's)
    constexpr int SIDE = 2;
#pragma unroll
    for (int t0 = 0; t0 < NT; t0 += SIDE) {
        uint32_t w[SIDE][4];
#pragma unroll
        for (int s = 0; s < SIDE; ++s) {
            const uint32_t from = at + (t0 + s) * 512 + n * 64;
            if (GP == 4) {
                const uint4 v = lds_128(from + ((j ^ (n >> 1)) & 3) * 16);
                w[s][0] = v.x; w[s][1] = v.y; w[s][2] = v.z; w[s][3] = v.w;
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) w[s][q] = lds_32(from + ((q ^ (n >> 1)) & 3) * 16 + 4 * j);
            }
        }
        int acc[SIDE][TILES][4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint32_t b[SIDE][2];
#pragma unroll
            for (int s = 0; s < SIDE; ++s) {
                b[s][0] = ((w[s][q] << 4) & 0xF0F0F0F0u) | one;
                b[s][1] = (w[s][q] & 0xF0F0F0F0u) | one;
            }
#pragma unroll
            for (int m = 0; m < TILES; ++m)
#pragma unroll
                for (int s = 0; s < SIDE; ++s) {
                    const uint32_t a[4] = {r.x[m][q].x, r.x[m][q].y, r.x[m][q].z, r.x[m][q].w};
                    if (q % GP == 0) mma_i8_first(acc[s][m], a, b[s][0], b[s][1]);
                    else mma_i8(acc[s][m], a, b[s][0], b[s][1]);
                }
            if (q % GP == GP - 1) {
#pragma unroll
                for (int s = 0; s < SIDE; ++s) {
                    const int t = t0 + s;
                    const uint2 sv = lds_64(as + (q / GP * NT * 8 + 8 * t + 2 * j) * 4);
                    const DsqPair scales = dsq_pair_of(__uint_as_float(sv.x), __uint_as_float(sv.y));
#pragma unroll
                    for (int m = 0; m < TILES; ++m) {
                        const DsqPair by = dsq_pair_mul(scales, dsq_pair_of(r.step[m], r.step[m]));
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            total[m][t][e] = dsq_pair_fma(dsq_pair_of((float)acc[s][m][2 * e], (float)acc[s][m][2 * e + 1]), by, total[m][t][e]);
                    }
                }
            }
        }
    }
}

constexpr int IN_WARPS = 8, OUT_WARPS = 4;

// A block's sums of a group: WC warps side by side on 16 columns of gate and other half each, IN_WARPS / WC along K.
template <int GP, int WC, int STAGES> struct In {
    using S = Stage<NT, GP>;
    static constexpr int KW = IN_WARPS / WC, RING = IN_WARPS * STAGES * S::BYTES, SUMS = IN_WARPS * NT * 512;
    static constexpr int BYTES = RING > SUMS ? RING : SUMS;

    static constexpr int TILES = 1;
    const MoeParams &p;
    const Members g;
    uint8_t *smem;
    int warp, lane, n, j, wk, c0, turns, to_turn, issued;
    uint32_t ring;
    Copies<NT, GP, STAGES> copies;

    __device__ __forceinline__ In(const MoeParams &p_, const Members &g_, uint8_t *smem_) : p(p_), g(g_), smem(smem_)
    {
        warp = threadIdx.x >> 5; lane = threadIdx.x & 31; n = lane >> 2; j = lane & 3;
        wk = warp / WC;
        c0 = (blockIdx.x * WC + warp % WC) * 16;
        turns = wk < p.chunks_in && (int)blockIdx.x * WC * 16 < p.I ? (p.chunks_in - wk - 1) / KW + 1 : 0;
        ring = smem_u32(smem) + (uint32_t)(warp * STAGES * S::BYTES);
        issued = 0;
        // columns 0 .. 15 are the gate's, 16 .. 31 the other half's
        auto row = [&](int c) { return (int64_t)g.expert * 2 * p.I + min(c0 + (c & 15), p.I - 1) + (c < 16 ? 0 : p.I); };
#pragma unroll
        for (int t = 0; t < NT; ++t) copies.w[t] = p.W_in + row(8 * t + n) * p.pitch_in;
        copies.scale = p.s_in + row(lane);
        copies.start(ring, wk, KW);
    }
    __device__ __forceinline__ void issue()
    {
        if (issued < turns) copies.next(p.pitch_in, (int64_t)p.E * 2 * p.I, p.groups_in, p.units_in, p.units_in_inv);
        ++issued;
        cp_async_commit();
    }
    // mid of (slot r of the group, column c of the block): gate and up are sums
    __device__ __forceinline__ void put(int r, int c, float gate, float up) const
    {
        const int at = blockIdx.x * WC * 16 + c;
        if (at >= p.chunks_out * 128) return;
        // (columns behind the last are zeros up to the end of the chunk)
        p.w.mid[(int64_t)g.slot(r) * p.chunks_out * 128 + at] = at < p.I ? activated(gate, p.act) * up : 0.f;
    }

    __device__ __forceinline__ void run()
    {
        Sources<TILES> from;
        Digits<TILES> d = {};
#pragma unroll
        for (int m = 0; m < TILES; ++m) {
            const int r = 4 * m + (n >> 1);
            const int token = r < g.n ? g.slot(r) / p.k : -1;
            if (token < 0) from.set(m, nullptr, nullptr);
            else from.set(m, p.w.x + (int64_t)token * p.chunks_in * 512, p.w.x_step + (int64_t)token * p.chunks_in);
        }
        if (turns > 0) from.load(wk, d);
        if (turns > 1) from.touch(wk + KW);
        DsqPair total[TILES][NT][2] = {};
#pragma unroll 1
        for (int i = 0; i < turns; ++i) {
            cp_async_wait<STAGES - 2>();
            __syncwarp();             // every lane's copies of this stage are here, and the last stage has been read
            issue();
            multiply_digits<TILES, NT, GP>(ring + (uint32_t)(i % STAGES * S::BYTES), d, total);
            if (i + 1 < turns) from.load(wk + (i + 1) * KW, d);
            if (i + 2 < turns) from.touch(wk + (i + 2) * KW);
        }
        // the warps' sums, added in a fixed order
        cp_async_wait<0>();
        __syncthreads();
        float4 *part = reinterpret_cast<float4 *>(smem);        // [IN_WARPS][TILES][NT][32]
#pragma unroll
        for (int m = 0; m < TILES; ++m)
#pragma unroll
            for (int t = 0; t < NT; ++t)
                reinterpret_cast<ulonglong2 *>(part)[((warp * TILES + m) * NT + t) * 32 + lane] = make_ulonglong2(total[m][t][0], total[m][t][1]);
        __syncthreads();
        const float unit = dsq_value_unit<DSQ_I8>(1);
        const float *sums = reinterpret_cast<const float *>(smem);
        for (int e = threadIdx.x; e < g.n * WC * 16; e += IN_WARPS * 32) {
            const int r = e / (WC * 16), c = e % (WC * 16), wc = c / 16;
            float both[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {                  // digit k
                    const int l = ((r & 3) * 2 + (k & 1)) * 4 + ((c & 7) >> 1);
                    const int at = (((r >> 2) * NT + 2 * u + ((c >> 3) & 1)) * 32 + l) * 4 + (k & 2) + (c & 1);
                    v[k] = 0.f;
#pragma unroll
                    for (int w = 0; w < KW; ++w) v[k] += sums[(w * WC + wc) * TILES * NT * 128 + at];
                }
                both[u] = __fmaf_rn(v[3], 0x1p-24f, __fmaf_rn(v[2], 0x1p-16f, __fmaf_rn(v[1], 0x1p-8f, v[0]))) * unit;
            }
            put(r, c, both[0], both[1]);
        }
        __syncthreads();
    }
};

template <int GP, int WC, int STAGES>
__global__ void __launch_bounds__(IN_WARPS * 32, 3) moe_in_kernel(const __grid_constant__ MoeParams p)
{
    extern __shared__ __align__(128) uint8_t smem[];
    // Where there are few slots their groups follow from the ids, which are older than the kernel ahead: the first codes are
    // on their way while that makes digits of x.
    Members g;
    int groups = -1;
    if (p.slots <= 32) {
        const Few few(p);
        if (few.fit) {
            groups = few.groups();
            if ((int)blockIdx.y < groups) {
                uint32_t slots;
                few.group(blockIdx.y, g.expert, slots);
                g.set(slots);
            }
        }
    }
    bool waited = groups < 0;
    if (waited) {
        grid_dependency_wait();
        grid_launch_dependents();
        // (what is there of a group that is not is not used)
        g = members_of(p.w, blockIdx.y);
        groups = *p.w.groups;
    }
    for (int i = blockIdx.y; i < groups; i += gridDim.y, g = members_of(p.w, min(i, groups - 1))) {
        In<GP, WC, STAGES> in(p, g, smem);
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s) in.issue();
        if (!waited) {
            grid_dependency_wait();
            grid_launch_dependents();
            waited = true;
        }
        in.run();
    }
    if (!waited) {
        grid_dependency_wait();
        grid_launch_dependents();
    }
}

// WC warps side by side on 32 columns each, OUT_WARPS / WC (and the cluster's blocks) along the chunks
template <int GP, int WC, int STAGES>
__global__ void __launch_bounds__(OUT_WARPS * 32, 5) moe_out_kernel(const __grid_constant__ MoeParams p, int cluster)
{
    constexpr int KW = OUT_WARPS / WC, WIDE = 8 * NT, COLS = WC * WIDE, THREADS = OUT_WARPS * 32;
    using S = Stage<NT, GP>;
    extern __shared__ __align__(128) uint8_t smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = lane >> 2, j = lane & 3;
    const int rank = cluster > 1 ? (int)cluster_ctarank() : 0;
    const int64_t b0 = (int64_t)(blockIdx.x / cluster) * COLS, c0 = b0 + warp % WC * WIDE;
    const uint32_t ring = smem_u32(smem) + (uint32_t)(warp * STAGES * S::BYTES);
    // [OUT_WARPS][T][WIDE]; the warp's own
    float *sums = reinterpret_cast<float *>(smem + OUT_WARPS * STAGES * S::BYTES), *mine = sums + warp * p.T * WIDE;
    for (int i = lane; i < p.T * WIDE; i += 32) mine[i] = 0.f;
    // Ahead of the wait: the slots, codes and scales are older than the kernel ahead (moe_mid_kernel; moe_in_kernel,
    // which moe_mid_kernel waits for before it lets this one start, waited for all that was in front of it).
    const int groups = *p.w.groups, chunks = p.chunks_out;
    // this warp's share of the chunks of all groups
    const int64_t all = (int64_t)groups * chunks;
    const int share = rank * KW + warp / WC, shares = cluster * KW;
    const int q0 = (int)(all * share / shares), q1 = (int)(all * (share + 1) / shares);
    int ig = q0 / chunks;                                       // group of the next copy
    Copies<NT, GP, STAGES> copies;
    auto columns_of = [&](int i) {
        const int64_t row0 = (int64_t)p.w.group[i].expert * p.H;
#pragma unroll
        for (int t = 0; t < NT; ++t) copies.w[t] = p.W_out + (row0 + min(c0 + 8 * t + n, (int64_t)p.H - 1)) * p.pitch_out;
        copies.scale = p.s_out + row0 + min(c0 + lane, (int64_t)p.H - 1);
    };
    auto issue = [&](int i) {
        if (i < q1) {
            copies.next(p.pitch_out, (int64_t)p.E * p.H, p.groups_out, p.units_out, p.units_out_inv);
            if (copies.chunk == chunks && i + 1 < q1) {
                const uint32_t to = copies.to;
                columns_of(++ig);
                copies.start(ring, 0, 1);
                copies.to = to;
            }
        }
        cp_async_commit();
    };
    if (q0 < q1) {
        columns_of(ig);
        copies.start(ring, q0 - ig * chunks, 1);
    }
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) issue(q0 + s);
    __syncwarp();
    grid_dependency_wait();
    grid_launch_dependents();

    Members g = {};
    Sources<1> from;
    Digits<1> d = {};
    int cg = q0 / chunks, cc = q0 - cg * chunks;                // of the chunk at hand
    auto rows_of = [&](int i) {
        g = members_of(p.w, i);
        d = {};
#pragma unroll
        for (int m = 0; m < 1; ++m) {
            const int r = 4 * m + (n >> 1);
            const int slot = r < g.n ? g.slot(r) : -1;
            if (slot < 0) from.set(m, nullptr, nullptr);
            else from.set(m, p.w.mid_rows + (int64_t)slot * chunks * 512, p.w.mid_step + (int64_t)slot * chunks);
        }
    };
    if (q0 < q1) {
        rows_of(cg);
        from.load(cc, d);
    }
    DsqPair total[1][NT][2] = {};
    // what a lane's digits n & 1 and (n & 1) + 2 stand for, in steps
    const float high = n & 1 ? 0x1p-8f : 1.f, low = n & 1 ? 0x1p-24f : 0x1p-16f;
#pragma unroll 1
    for (int i = q0; i < q1; ++i) {
        cp_async_wait<STAGES - 2>();
        __syncwarp();
        issue(i + STAGES - 1);
        const uint32_t at = ring + (uint32_t)((i - q0) % STAGES * S::BYTES);
        multiply_digits<1, NT, GP>(at, d, total);
        if (++cc < chunks && i + 1 < q1) {
            from.load(cc, d);
            if (cc + 1 < chunks && i + 2 < q1) from.touch(cc + 1);
            continue;
        }
        // the group's sums to the tokens' rows, one slot after the other (two may be the same token's)
#pragma unroll
        for (int m = 0; m < 1; ++m) {
            if (4 * m >= g.n) break;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float h0, h1, l0, l1;
                dsq_halves(total[m][t][0], h0, h1);
                dsq_halves(total[m][t][1], l0, l1);
                h0 = __fmaf_rn(l0, low, h0 * high);
                h1 = __fmaf_rn(l1, low, h1 * high);
                h0 += __shfl_xor_sync(~0u, h0, 4);
                h1 += __shfl_xor_sync(~0u, h1, 4);
                total[m][t][0] = dsq_pair_of(h0, h1);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (4 * m + r >= g.n) break;
                if (n == 2 * r) {
                    const int slot = g.slot(4 * m + r), token = slot / p.k;
                    const float w = p.weights[slot];
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        float2 *to = reinterpret_cast<float2 *>(mine + token * WIDE + 8 * t + 2 * j);
                        float2 v = *to;
                        float h0, h1;
                        dsq_halves(total[m][t][0], h0, h1);
                        v.x = __fmaf_rn(h0, w, v.x);
                        v.y = __fmaf_rn(h1, w, v.y);
                        *to = v;
                    }
                }
                __syncwarp();
            }
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e) total[m][t][e] = 0ull;
        }
        if (cc == chunks) {
            cc = 0;
            ++cg;
        }
        if (i + 1 < q1) {
            rows_of(cg);
            from.load(cc, d);
            if (cc + 1 < chunks && i + 2 < q1) from.touch(cc + 1);
        }
    }
    cp_async_wait<0>();
    __syncthreads();
    // the sums of the warps along the chunks, into the first one's place
    for (int e = threadIdx.x; e < p.T * COLS; e += THREADS) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < KW; ++w) s += sums[w * p.T * COLS + e];
        if (KW > 1) sums[e] = s;
    }
    if (cluster > 1) cluster_sync_all();
    else __syncthreads();
    const float unit = dsq_value_unit<DSQ_I8>(1);
    for (int e = rank * THREADS + threadIdx.x; e < p.T * COLS; e += cluster * THREADS) {
        float s = 0.f;
        if (cluster == 1) s = sums[e];
        else
            for (int c = 0; c < cluster; ++c) s += __uint_as_float(ld_cluster_32(map_to_cta(smem_u32(sums + e), c)));
        // (a row of 32 columns of each of the warps side by side)
        const int wc = e / (p.T * WIDE), token = e / WIDE - wc * p.T;
        const int64_t col = b0 + wc * WIDE + e % WIDE;
        if (col >= p.H) continue;
        const int64_t to = (int64_t)token * p.H + col;
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
constexpr int IN_STAGES = 3, OUT_STAGES = 4, IN_SIDE = 2, OUT_SIDE = 1;     // warps side by side

template <int XT, int GP> int launch_prepare(const MoeParams &p, cudaStream_t s)
{
    const int blocks = 1 + (p.T * p.chunks_in + PREPARE_WARPS - 1) / PREPARE_WARPS;
    return dsq_launch(moe_prepare_kernel<XT, GP == 4>, dim3(blocks), dim3(PREPARE_WARPS * 32), 0, s, dsq_launch_hooks().pdl, 0, p);
}

template <int GP> int launch_in(const MoeParams &p, cudaStream_t s)
{
    constexpr int bytes = In<GP, IN_SIDE, IN_STAGES>::BYTES, cols = IN_SIDE * 16;
    static_assert(bytes <= 74 * 1024, "shared memory");
    static std::atomic<unsigned long long> configured{0};
    const auto kernel = moe_in_kernel<GP, IN_SIDE, IN_STAGES>;
    const int st = dsq_allow_smem((const void *)kernel, bytes, &configured);
    if (st) return st;
    // (to the end of the last chunk: zeros)
    const dim3 grid((unsigned)((p.chunks_out * 128 + cols - 1) / cols), (unsigned)p.groups_most());
    return dsq_launch(kernel, grid, dim3(IN_WARPS * 32), (size_t)bytes, s, dsq_launch_hooks().pdl, 0, p);
}

template <int GP> int launch_out(const MoeParams &p, cudaStream_t s)
{
    constexpr int ring = OUT_WARPS * OUT_STAGES * Stage<NT, GP>::BYTES, row = OUT_WARPS * 8 * NT * 4, cols = OUT_SIDE * 8 * NT;
    static_assert(ring + PASS_TOKENS * row <= 200 * 1024, "shared memory");
    static std::atomic<unsigned long long> configured{0};
    const auto kernel = moe_out_kernel<GP, OUT_SIDE, OUT_STAGES>;
    const int st = dsq_allow_smem((const void *)kernel, ring + PASS_TOKENS * row, &configured);
    if (st) return st;
    const int tiles = (p.H + cols - 1) / cols, sms = dsq_sm_count() > 0 ? dsq_sm_count() : 148;
    int cluster = 4 * sms / tiles;
    cluster = cluster < 1 ? 1 : cluster > 8 ? 8 : cluster;
    return dsq_launch(kernel, dim3((unsigned)(tiles * cluster)), dim3(OUT_WARPS * 32), (size_t)(ring + p.T * row), s,
                      dsq_launch_hooks().pdl, cluster, p, cluster);
}

template <int XT, int GP> int run_in(const MoeParams &p, cudaStream_t s)
{
    const int st = launch_prepare<XT, GP>(p, s);
    return st ? st : launch_in<GP>(p, s);
}
template <int GP> int run_out(const MoeParams &p, cudaStream_t s)
{
    const int st = dsq_launch(moe_mid_kernel<GP == 4>, dim3((p.slots * p.chunks_out + PREPARE_WARPS - 1) / PREPARE_WARPS),
                              dim3(PREPARE_WARPS * 32), 0, s, dsq_launch_hooks().pdl, 0, p);
    return st ? st : launch_out<GP>(p, s);
}
int run_digits(const MoeParams &p, int x_type, int gp_in, int gp_out, cudaStream_t s)
{
    int st;
    if (x_type == DSQ_BF16) st = gp_in == 4 ? run_in<DSQ_BF16, 4>(p, s) : gp_in == 2 ? run_in<DSQ_BF16, 2>(p, s) : run_in<DSQ_BF16, 1>(p, s);
    else st = gp_in == 4 ? run_in<DSQ_F16, 4>(p, s) : gp_in == 2 ? run_in<DSQ_F16, 2>(p, s) : run_in<DSQ_F16, 1>(p, s);
    return st ? st : gp_out == 4 ? run_out<4>(p, s) : gp_out == 2 ? run_out<2>(p, s) : run_out<1>(p, s);
}

int chunks_of(int64_t K) { return (int)((K + 127) / 128); }

// Lays the workspace out behind its first bytes, for either form; returns its size.
size_t lay_out(Work &w, char *base, int T, int slots, int H, int chunks_in, int chunks_out)
{
    size_t at = DSQ_WS_BYTES;
    auto take = [&](size_t bytes) {
        char *p = base + at;
        at += (bytes + 255) / 256 * 256;
        return p;
    };
    const size_t mid = (size_t)slots * chunks_out * 512, part = (size_t)slots * H * 4;
    w.groups = (int *)take(4);
    w.group = (Group *)take((size_t)slots * sizeof(Group));
    w.x_step = (float *)take((size_t)T * chunks_in * 4);
    w.mid_step = (float *)take((size_t)slots * chunks_out * 4);
    w.x = (uint8_t *)take((size_t)T * chunks_in * 512);
    w.mid_rows = (uint8_t *)take((size_t)slots * chunks_out * 512);
    w.mid = (float *)take(mid > part ? mid : part);
    w.part = w.mid;
    return at;
}

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

size_t dsq_moe_workspace_bytes(int64_t T, int64_t H, int64_t I, int k)
{
    if (T <= 0 || H <= 0 || H > DSQ_GROUPS_MAX_K || I <= 0 || I > DSQ_GROUPS_MAX_K || k <= 0 || k > MAX_TOP) return DSQ_WS_BYTES;
    const int tokens = (int)(T < PASS_TOKENS ? T : PASS_TOKENS);
    Work w;
    return lay_out(w, nullptr, tokens, tokens * k, (int)H, chunks_of(H), chunks_of(I));
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
    if (ws_bytes < dsq_moe_workspace_bytes(T, H, I, k)) return DSQ_ERR_SIZE;
    const int64_t g_in = group_of_row(H, group), g_out = group_of_row(I, group);
    const int gp_in = dsq_group_pieces(g_in), gp_out = dsq_group_pieces(g_out);
    MoeParams p;
    p.W_in = (const uint8_t *)W_in; p.W_out = (const uint8_t *)W_out;
    p.s_in = scales_in; p.s_out = scales_out;
    p.H = (int)H; p.I = (int)I; p.E = (int)E; p.k = k;
    p.pitch_in = (int)dsq_row_pitch(H, 4); p.pitch_out = (int)dsq_row_pitch(I, 4);
    p.chunks_in = chunks_of(H); p.chunks_out = chunks_of(I);
    p.groups_in = (int)dsq_group_count(H, g_in); p.groups_out = (int)dsq_group_count(I, g_out);
    set_units(g_in, gp_in, &p.units_in, &p.units_in_inv);
    set_units(g_out, gp_out, &p.units_out, &p.units_out_inv);
    p.odd = w_offset == 0.5f; p.act = activation; p.y_type = y_type;
    cudaStream_t s = (cudaStream_t)stream;
    const int64_t y_size = y_type == DSQ_F32 ? 4 : 2;
    for (int64_t t = 0; t < T; t += PASS_TOKENS) {
        p.T = (int)(T - t < PASS_TOKENS ? T - t : PASS_TOKENS);
        p.slots = p.T * k;
        // Digits where few experts can be expected to have several slots, and where no code is 0 (see above): at 54 sizes
        // within 14 % of the faster form, 1.5 % on average.  4096 to 2048, 8 experts, two a token: 2 tokens 20.1 us on digits, 26.8 on
        // 16 bits; 5 tokens 32.7 and 36.2; 8 tokens 36.2 and 36.8; 48 tokens 107 and 56.  4096 to 1024, 64 experts, four
        // a token: 4 tokens 32.1 and 35.4; 24 tokens 85.7 and 91.4; 32 tokens 97.6 and 100.2; 48 tokens 145 and 117.
        const bool digits = p.odd && (p.T <= 4 || 2 * p.slots <= 3 * p.E);
        // On 16 bits sixteen slots share an expert's codes where it can be expected to have more than five, with two blocks an SM
        // instead of three: 48 tokens of 4096 to 2048, 8 experts, two a token, 56 us, 71 with eight; of 4096 to 1024, 64
        // experts, four a token, 129 us and 117.
        p.scaled = !digits && p.odd && x_type == DSQ_BF16;
        p.rows = digits ? 4 : p.slots <= 5 * p.E ? 8 : 16;
        lay_out(p.w, (char *)workspace, p.T, p.slots, p.H, p.chunks_in, p.chunks_out);
        p.X = (const uint8_t *)X + t * H * 2;
        p.ids = ids + t * k; p.weights = weights + t * k;
        p.residual = residual ? (const char *)residual + t * H * y_size : nullptr;
        p.Y = (char *)Y + t * H * y_size;
        st = digits ? run_digits(p, x_type, gp_in, gp_out, s) : run_wide(p, x_type, gp_in, gp_out, s);
        if (st) return st;
    }
    return DSQ_OK;
}

}  // extern "C"
