// A layer of experts (dsq_moe.cu states it) where experts have several tokens: on 16 bits.
//
// On digits every four slots cost an instruction of 8 clocks a scheduler for a word of codes; here a word costs ten or
// twelve operations, but then two instructions take up to sixteen slots.
//   * The weights are the 16 rows of an instruction, the slots its 8 columns: a lane has one slot's elements
//     (half the registers of digits) and sums of 16 columns by 8 slots in four registers.
//   * Codes become bf16 or fp16 pairs, x is rearranged once, so that 16 bytes are a word's elements in the
//     operand's order: products are exact and added in binary32.  Rows of bf16 go as fp16 times a power of two where no code is
//     0: exact down to 2^-31 of a token's largest element, off by 2^-39 of it (or 2^-151) below, far below the sums' rounding
//     (16 tokens of 4096 to 1024, four of 64 experts: 81 us with twelve operations a word, 73.6 with ten).
//   * mid, in binary32 first, goes as two fp16 numbers, 22 bits, on a power of two of its own for each slot, its largest below
//     2^15; they are two rows of elements, so that four slots fill an instruction's columns there.  (One number, 11 bits, is 12 us
//     faster below, but Y then shows its rounding wherever a residual takes most of the sum away, and other numbers of tokens in a
//     call, which go on digits, change Y by as much.)
//   * moe_wide_kernel does both products: a block has 4 warps side by side on 32 columns each (16 of gate and
//     other half; or 32 of y) and 2 along K; the warps' sums are added in a fixed order.  What each slot adds to its
//     token goes to the workspace, moe_combine_kernel adds it slot by slot.
// 64 tokens of 4096 to 2048, four of 32 experts (429 MB of codes and scales): 146 us, 2.9 TB/s.  No unit is saturated (issue slots
// 53 % and 41 %, tensor pipe 32 % and 34 %, DRAM 42 % and 28 % in the two products): four warps a scheduler (128 registers)
// do not cover the loads of their rows from L1 and the chains of products; without those loads the second product takes two thirds.
#include "dsq_moe.cuh"

using namespace dsq_moe;

namespace {

constexpr int WARPS = 8, WC = 4, KW = WARPS / WC, THREADS = WARPS * 32, STAGES = 4;

// where pair i of the code word `word` of a chunk lies in a row's 256 bytes: lane j's word q is 4 j + q where no
// group's end cuts the chunk (WHOLE), else j + 4 q
template <bool WHOLE> __device__ __forceinline__ int place_of(int word)
{
    const int j = WHOLE ? word >> 2 : word & 3, q = WHOLE ? word & 3 : word >> 2;
    return q * 64 + j * 16;
}

// block 0: the slots; the others' warps a chunk of a token each: elements i and i + 4 of a word side by side
constexpr int PREPARE_WARPS = 8;
template <bool WHOLE> __global__ void __launch_bounds__(PREPARE_WARPS * 32) moe_wide_prepare_kernel(const __grid_constant__ MoeParams p)
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
    uint2 v = make_uint2(0u, 0u);
    if (k < p.H) v = *reinterpret_cast<const uint2 *>(p.X + ((int64_t)t * p.H + k) * 2);     // (H is a multiple of 8)
    // the other half of the word, and pairs of both
    const uint2 o = make_uint2(__shfl_xor_sync(~0u, v.x, 1), __shfl_xor_sync(~0u, v.y, 1));
    uint8_t *to = p.w.x + (int64_t)i * 256 + place_of<WHOLE>(lane >> 1);
    if (lane & 1) *reinterpret_cast<uint2 *>(to + 8) = make_uint2(__byte_perm(o.y, v.y, 0x5410), __byte_perm(o.y, v.y, 0x7632));
    else *reinterpret_cast<uint2 *>(to) = make_uint2(__byte_perm(v.x, o.x, 0x5410), __byte_perm(v.x, o.x, 0x7632));
}

// The power of two that brings the largest of a row below 2^15 (the smallest numbers' rows as far as binary32 has
// powers of two), and what 1 stands for then; a block has the largest of each thread's elements, and whether one is
// infinite or NaN.
__device__ __forceinline__ float block_scale(float m, bool bad, float *step)
{
    __shared__ float most[8];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
    if ((threadIdx.x & 31) == 0) most[threadIdx.x >> 5] = m;
    bad = __syncthreads_or(bad);
#pragma unroll
    for (int w = 0; w < 8; ++w) m = fmaxf(m, most[w]);
    const int e = (int)(__float_as_uint(m) >> 23), up = min(141 - e, 126);
    if (threadIdx.x == 0) *step = __uint_as_float(bad ? 0x7FC00000u : (uint32_t)(127 - up) << 23);
    return __uint_as_float((uint32_t)(127 + up) << 23);
}

// the same of bf16 as fp16 (scaled): block 1 + t has token t
template <bool WHOLE> __global__ void __launch_bounds__(256) moe_wide_prepare_scaled_kernel(const __grid_constant__ MoeParams p)
{
    __shared__ Sorting sorting;
    grid_dependency_wait();
    grid_launch_dependents();
    if (blockIdx.x == 0) {
        sort_slots(p, sorting);
        return;
    }
    const int t = blockIdx.x - 1, words = p.chunks_in * 16;
    const uint4 *row = reinterpret_cast<const uint4 *>(p.X + (int64_t)t * p.H * 2);
    float m = 0.f;
    bool bad = false;
    for (int i = threadIdx.x; 8 * i < p.H; i += 256) {
        float f[8];
        dsq_unpack8(dsq_load8(reinterpret_cast<const __nv_bfloat16 *>(row + i)), f);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            m = fmaxf(m, fabsf(f[e]));
            bad = bad || !(fabsf(f[e]) <= 3.402823466e38f);
        }
    }
    const float by = block_scale(m, bad, p.w.x_step + t);
    for (int i = threadIdx.x; i < words; i += 256) {
        float f[8] = {};
        if (8 * i < p.H) dsq_unpack8(dsq_load8(reinterpret_cast<const __nv_bfloat16 *>(row + i)), f);
        uint32_t v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const __half2 h = __floats2half2_rn(f[k] * by, f[k + 4] * by);
            v[k] = *reinterpret_cast<const uint32_t *>(&h);
        }
        *reinterpret_cast<uint4 *>(p.w.x + ((int64_t)t * p.chunks_in + (i >> 4)) * 256 + place_of<WHOLE>(i & 15)) =
            make_uint4(v[0], v[1], v[2], v[3]);
    }
}

// mid's rows, a block a slot (of slots without an expert: of whatever lies there)
template <bool WHOLE> __global__ void __launch_bounds__(256) moe_wide_mid_kernel(const __grid_constant__ MoeParams p)
{
    const int slot = blockIdx.x;
    grid_dependency_wait();
    grid_launch_dependents();
    const float *mid = p.w.mid + (int64_t)slot * p.chunks_out * 128;
    const int words = p.chunks_out * 16;
    float m = 0.f;
    bool bad = false;
    for (int i = threadIdx.x; i < words * 2; i += 256) {
        const float4 v = reinterpret_cast<const float4 *>(mid)[i];
        const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            m = fmaxf(m, fabsf(f[e]));
            bad = bad || !(fabsf(f[e]) <= 3.402823466e38f);
        }
    }
    const float by = block_scale(m, bad, p.w.mid_step + slot);
    uint8_t *rows = p.w.mid_rows + (int64_t)slot * p.chunks_out * 512;
    for (int i = threadIdx.x; i < words; i += 256) {
        const float4 a = reinterpret_cast<const float4 *>(mid)[2 * i], b = reinterpret_cast<const float4 *>(mid)[2 * i + 1];
        const float f[4][2] = {{a.x, b.x}, {a.y, b.y}, {a.z, b.z}, {a.w, b.w}};
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float x = f[k][0] * by, y = f[k][1] * by;
            const __half2 h = __floats2half2_rn(x, y);
            const float2 back = __half22float2(h);
            const __half2 l = __floats2half2_rn(x - back.x, y - back.y);
            hi[k] = *reinterpret_cast<const uint32_t *>(&h);
            lo[k] = *reinterpret_cast<const uint32_t *>(&l);
        }
        // (a line for the words of four lanes: 64 bytes of first numbers, 64 of second ones)
        const int place = place_of<WHOLE>(i & 15);
        uint8_t *to = rows + (int64_t)(i >> 4) * 512 + (place >> 6) * 128 + (place & 63);
        *reinterpret_cast<uint4 *>(to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        *reinterpret_cast<uint4 *>(to + 64) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
}

// ---- products
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
// the same on sums of zero
template <int XT> __device__ __forceinline__ void mma_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if (XT == DSQ_BF16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
            "{%8, %9}, {%10, %10, %10, %10};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
            "{%8, %9}, {%10, %10, %10, %10};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

// A word of codes as operands' pairs: of elements i and i + 4 each.  For fp16 two of the four fields lie in the
// mantissa at once, at its bits 1 to 4 and 5 to 8 of 32 and 2: two shifts instead of four (10 operations a word; bf16 has no
// room for a second field: 12).
template <int XT> struct Unpack {
    uint32_t base;
    __device__ __forceinline__ Unpack(int odd) : base(dsq_value_base<XT>(odd)) {}
    __device__ __forceinline__ void operator()(uint32_t w, uint32_t (&v)[4]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = dsq_value_pair<XT>(w, i, base);
    }
};
template <> struct Unpack<DSQ_F16> {
    uint32_t low, high;               // 32 and 2, and 7.5 / 16 or 8 / 16 beside
    __device__ __forceinline__ Unpack(int odd) : low(odd ? 0x500F500Fu : 0x50105010u), high(odd ? 0x40F040F0u : 0x41004100u) {}
    __device__ __forceinline__ void operator()(uint32_t w, uint32_t (&v)[4]) const
    {
        const uint32_t y[2] = {w << 1, w >> 7};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t mask = i & 1 ? 0x01E001E0u : 0x001E001Eu, flip = i & 1 ? 0x41004100u : 0x50105010u;
            const uint32_t less = i & 1 ? high : low;
            uint32_t f;
            asm("lop3.b32 %0, %1, %2, %3, 0x6a;" : "=r"(f) : "r"(y[i >> 1]), "r"(mask), "r"(flip));
            const __half2 r = __hsub2(*reinterpret_cast<const __half2 *>(&f), *reinterpret_cast<const __half2 *>(&less));
            v[i] = *reinterpret_cast<const uint32_t *>(&r);
        }
    }
};

// What a lane has of a chunk's rows: of each tile of eight slots the elements of slot n beside its own words of codes.
template <int TILES> struct Elements { uint4 x[TILES][4]; };

// total[h][m] += scale (sum of v x) of a chunk: rows n and n + 8 of half h of the 32 columns, slots 2 j and 2 j + 1 of tile m
template <int XT, int TILES, int GP>
__device__ __forceinline__ void multiply(uint32_t at, const Unpack<XT> &unpack, const Elements<TILES> &r, DsqPair (&total)[2][TILES][2])
{
    const int lane = threadIdx.x & 31, n = lane >> 2, j = lane & 3;
    const uint32_t as = at + Stage<NT, GP>::W_BYTES + n * 4;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t w[2][4];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint32_t from = at + (2 * h + s) * 512 + n * 64;
            if (GP == 4) {
                const uint4 v = lds_128(from + ((j ^ (n >> 1)) & 3) * 16);
                w[s][0] = v.x; w[s][1] = v.y; w[s][2] = v.z; w[s][3] = v.w;
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) w[s][q] = lds_32(from + ((q ^ (n >> 1)) & 3) * 16 + 4 * j);
            }
        }
        float acc[TILES][4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint32_t a[2][4];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                uint32_t v[4];
                unpack(w[s][q], v);
#pragma unroll
                for (int i = 0; i < 4; ++i) a[i >> 1][(i & 1) * 2 + s] = v[i];
            }
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int m = 0; m < TILES; ++m) {
                    const uint32_t b0 = s ? r.x[m][q].z : r.x[m][q].x, b1 = s ? r.x[m][q].w : r.x[m][q].y;
                    if (q % GP == 0 && s == 0) mma_first<XT>(acc[m], a[s], b0, b1);
                    else mma<XT>(acc[m], a[s], b0, b1);
                }
            if (q % GP == GP - 1) {
                const uint32_t from = as + (q / GP * NT * 8 + 16 * h) * 4;
                const float s0 = __uint_as_float(lds_32(from)), s1 = __uint_as_float(lds_32(from + 32));
#pragma unroll
                for (int m = 0; m < TILES; ++m) {
                    total[h][m][0] = dsq_pair_fma(dsq_pair_of(acc[m][0], acc[m][1]), dsq_pair_of(s0, s0), total[h][m][0]);
                    total[h][m][1] = dsq_pair_fma(dsq_pair_of(acc[m][2], acc[m][3]), dsq_pair_of(s1, s1), total[h][m][1]);
                }
            }
        }
    }
}

// The same of slots whose elements are two numbers each, the first in row 2 i of a tile of four slots, the second in row 2 i + 1: a lane
// has both sums of slot j, and adds them.  Elements come word by word, WORDS (2 or 4) less one ahead: pieces[q % WORDS] has those of
// word q when its turn comes, fetch(q, to) brings those of word q (from 4 on the next chunk's).
template <int TILES> struct Piece { uint4 x[TILES]; };
template <int XT, int TILES, int GP, int WORDS, class F>
__device__ __forceinline__ void multiply_both(uint32_t at, const Unpack<XT> &unpack, Piece<TILES> (&pieces)[WORDS], DsqPair (&total)[2][TILES], F fetch)
{
    const int lane = threadIdx.x & 31, n = lane >> 2, j = lane & 3;
    const uint32_t as = at + Stage<NT, GP>::W_BYTES + n * 4;
    uint32_t w[4][4];
    if (GP == 4) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const uint4 v = lds_128(at + t * 512 + n * 64 + ((j ^ (n >> 1)) & 3) * 16);
            w[t][0] = v.x; w[t][1] = v.y; w[t][2] = v.z; w[t][3] = v.w;
        }
    }
    float acc[2][TILES][4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        fetch(q + WORDS - 1, pieces[(q + WORDS - 1) % WORDS]);
        const Piece<TILES> &r = pieces[q % WORDS];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t a[2][4];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                uint32_t v[4];
                if (GP != 4) w[2 * h + s][q] = lds_32(at + (2 * h + s) * 512 + n * 64 + ((q ^ (n >> 1)) & 3) * 16 + 4 * j);
                unpack(w[2 * h + s][q], v);
#pragma unroll
                for (int i = 0; i < 4; ++i) a[i >> 1][(i & 1) * 2 + s] = v[i];
            }
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int m = 0; m < TILES; ++m) {
                    const uint32_t b0 = s ? r.x[m].z : r.x[m].x, b1 = s ? r.x[m].w : r.x[m].y;
                    if (q % GP == 0 && s == 0) mma_first<XT>(acc[h][m], a[s], b0, b1);
                    else mma<XT>(acc[h][m], a[s], b0, b1);
                }
            if (q % GP == GP - 1) {
                const uint32_t from = as + (q / GP * NT * 8 + 16 * h) * 4;
                const DsqPair scales = dsq_pair_of(__uint_as_float(lds_32(from)), __uint_as_float(lds_32(from + 32)));
#pragma unroll
                for (int m = 0; m < TILES; ++m)
                    total[h][m] = dsq_pair_fma(dsq_pair_of(acc[h][m][0] + acc[h][m][1], acc[h][m][2] + acc[h][m][3]), scales, total[h][m]);
            }
        }
    }
}

template <bool OUT, int XT, int GP> struct Wide {
    using S = Stage<NT, GP>;
    static constexpr int RING = WARPS * STAGES * S::BYTES, SUMS = WARPS * 2 * 2 * 512;
    static constexpr int BYTES = RING > SUMS ? RING : SUMS;

    const MoeParams &p;
    const Group *group;
    uint8_t *smem;
    int expert, slots, warp, lane, n, j, wk, c0, chunks, turns, issued;
    uint32_t ring;
    Copies<NT, GP, STAGES> copies;

    __device__ __forceinline__ Wide(const MoeParams &p_, const Group *group_, int expert_, int slots_, uint8_t *smem_)
        : p(p_), group(group_), smem(smem_), expert(expert_), slots(slots_)
    {
        warp = threadIdx.x >> 5; lane = threadIdx.x & 31; n = lane >> 2; j = lane & 3;
        wk = warp / WC;
        // columns of the warp: 16 of the gate and the same of the other half, or 32 of y
        c0 = (blockIdx.x * WC + warp % WC) * (OUT ? 32 : 16);
        chunks = OUT ? p.chunks_out : p.chunks_in;
        const int columns = OUT ? p.H : p.I;
        turns = wk < chunks && (int)blockIdx.x * WC * (OUT ? 32 : 16) < columns ? (chunks - wk - 1) / KW + 1 : 0;
        ring = smem_u32(smem) + (uint32_t)(warp * STAGES * S::BYTES);
        issued = 0;
        auto row = [&](int c) {
            if (OUT) return (int64_t)expert * p.H + min(c0 + c, p.H - 1);
            return (int64_t)expert * 2 * p.I + min(c0 + (c & 15), p.I - 1) + (c < 16 ? 0 : p.I);
        };
#pragma unroll
        for (int t = 0; t < NT; ++t)
            copies.w[t] = (OUT ? p.W_out : p.W_in) + row(8 * t + n) * (OUT ? p.pitch_out : p.pitch_in);
        copies.scale = (OUT ? p.s_out : p.s_in) + row(lane);
        copies.start(ring, wk, KW);
    }
    __device__ __forceinline__ void issue()
    {
        if (issued < turns) {
            if (OUT) copies.next(p.pitch_out, (int64_t)p.E * p.H, p.groups_out, p.units_out, p.units_out_inv);
            else copies.next(p.pitch_in, (int64_t)p.E * 2 * p.I, p.groups_in, p.units_in, p.units_in_inv);
        }
        ++issued;
        cp_async_commit();
    }

    // this warp's turns: codes of each as they come
    template <class F> __device__ __forceinline__ void each_turn(F f)
    {
#pragma unroll 1
        for (int i = 0; i < turns; ++i) {
            cp_async_wait<STAGES - 2>();
            __syncwarp();             // every lane's copies of this stage are here, and the last stage has been read
            issue();
            f(i, ring + (uint32_t)(i % STAGES * S::BYTES));
        }
        cp_async_wait<0>();
        __syncthreads();
    }
    // (a line a lane into L1, ahead of the loads, which would wait for L2 with every register taken; rows of `lines` lines a chunk)
    template <int TILES> __device__ __forceinline__ void touch(const uint8_t *(&x)[TILES], int chunk, int lines) const
    {
#pragma unroll
        for (int m = 0; m < TILES; ++m)
            if (x[m] && j < lines) {
                uint32_t none;
                asm volatile("ld.global.u32 %0, [%1];" : "=r"(none) : "l"(x[m] + (int64_t)chunk * 128 * lines + j * 112));
            }
    }

    // the first product of up to 8 TILES slots
    template <int TILES> __device__ __forceinline__ void run_in()
    {
        const Unpack<XT> unpack(p.odd);
        const uint8_t *x[TILES];
        Elements<TILES> r = {};
#pragma unroll
        for (int m = 0; m < TILES; ++m)
            x[m] = 8 * m + n < slots ? p.w.x + (int64_t)(group->slot[8 * m + n] / p.k) * chunks * 256 + 16 * j : nullptr;
        // (rows of no slot stay zeros)
        auto load = [&](int chunk) {
#pragma unroll
            for (int m = 0; m < TILES; ++m)
                if (x[m]) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) r.x[m][q] = load_16(x[m] + (int64_t)chunk * 256 + 64 * q);
                }
        };
        if (turns > 0) load(wk);
        if (turns > 1) touch(x, wk + KW, 2);
        DsqPair total[2][TILES][2] = {};
        each_turn([&](int i, uint32_t at) {
            multiply<XT, TILES, GP>(at, unpack, r, total);
            if (i + 1 < turns) load(wk + (i + 1) * KW);
            if (i + 2 < turns) touch(x, wk + (i + 2) * KW, 2);
        });
        // the warps' sums, added in a fixed order
        ulonglong2 *part = reinterpret_cast<ulonglong2 *>(smem);       // [WARPS][2][TILES][32]
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int m = 0; m < TILES; ++m)
                part[((warp * 2 + h) * TILES + m) * 32 + lane] = make_ulonglong2(total[h][m][0], total[h][m][1]);
        __syncthreads();
        const float unit = dsq_value_unit<XT>(p.odd);
        const float *sums = reinterpret_cast<const float *>(smem);
        // the sum of slot i and column c of half h of the wc-th warp's
        auto sum = [&](int wc, int h, int c, int i) {
            const int at = ((h * TILES + (i >> 3)) * 32 + (c & 7) * 4 + ((i & 7) >> 1)) * 4 + 2 * (c >> 3) + (i & 1);
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < KW; ++w) v += sums[(w * WC + wc) * 2 * TILES * 128 + at];
            return v;
        };
        for (int e = threadIdx.x; e < slots * WC * 16; e += THREADS) {
            const int s = e / (WC * 16), c = e % (WC * 16), col = blockIdx.x * WC * 16 + c;
            if (col >= chunks_of_mid()) continue;
            // (columns behind the last are zeros up to the end of the chunk)
            const int slot = group->slot[s];
            const float of_x = p.scaled ? unit * p.w.x_step[slot / p.k] : unit;
            const float gate = sum(c >> 4, 0, c & 15, s) * of_x, up = sum(c >> 4, 1, c & 15, s) * of_x;
            p.w.mid[(int64_t)slot * chunks_of_mid() + col] = col < p.I ? activated(gate, p.act) * up : 0.f;
        }
        __syncthreads();
    }

    // the second product of up to 4 TILES slots, WORDS words of elements on their way
    template <int TILES, int WORDS> __device__ __forceinline__ void run_out()
    {
        const Unpack<XT> unpack(p.odd);
        const uint8_t *x[TILES];
        Piece<TILES> pieces[WORDS] = {};
#pragma unroll
        for (int m = 0; m < TILES; ++m)
            x[m] = 4 * m + (n >> 1) < slots ? p.w.mid_rows + (int64_t)group->slot[4 * m + (n >> 1)] * chunks * 512 + 64 * (n & 1) + 16 * j : nullptr;
        // (rows of no slot stay zeros)
        auto fetch = [&](int chunk, int q, Piece<TILES> &to) {
#pragma unroll
            for (int m = 0; m < TILES; ++m)
                if (x[m]) to.x[m] = load_16(x[m] + (int64_t)chunk * 512 + 128 * q);
        };
        if (turns > 0) {
#pragma unroll
            for (int q = 0; q < WORDS - 1; ++q) fetch(wk, q, pieces[q]);
        }
        if (turns > 1) touch(x, wk + KW, 4);
        DsqPair total[2][TILES] = {};
        each_turn([&](int i, uint32_t at) {
            multiply_both<XT, TILES, GP, WORDS>(at, unpack, pieces, total, [&](int q, Piece<TILES> &to) {
                if (q < 4) fetch(wk + i * KW, q, to);
                else if (i + 1 < turns) fetch(wk + (i + 1) * KW, q - 4, to);
            });
            if (i + 2 < turns) touch(x, wk + (i + 2) * KW, 4);
        });
        // the warps' sums, added in a fixed order
        DsqPair *part = reinterpret_cast<DsqPair *>(smem);             // [WARPS][2][TILES][32]
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int m = 0; m < TILES; ++m) part[((warp * 2 + h) * TILES + m) * 32 + lane] = total[h][m];
        __syncthreads();
        const float unit = dsq_value_unit<XT>(p.odd);
        const float *sums = reinterpret_cast<const float *>(smem);
        for (int e = threadIdx.x; e < slots * WC * 32; e += THREADS) {
            const int s = e / (WC * 32), c = e % (WC * 32), col = blockIdx.x * WC * 32 + c, wc = c >> 5, h = c >> 4 & 1;
            if (col >= p.H) continue;
            const int at = ((h * TILES + (s >> 2)) * 32 + (c & 7) * 4 + (s & 3)) * 2 + (c >> 3 & 1);
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < KW; ++w) v += sums[(w * WC + wc) * 2 * TILES * 64 + at];
            const int slot = group->slot[s];
            p.w.part[(int64_t)slot * p.H + col] = v * unit * p.w.mid_step[slot] * p.weights[slot];
        }
        __syncthreads();
    }
    __device__ __forceinline__ int chunks_of_mid() const { return p.chunks_out * 128; }
};

// MOST: eights of slots of a group
template <bool OUT, int XT, int GP, int MOST>
__global__ void __launch_bounds__(THREADS, MOST == 1 ? 3 : 2) moe_wide_kernel(const __grid_constant__ MoeParams p)
{
    extern __shared__ __align__(128) uint8_t smem[];
    // (the second product: slots, codes and scales are older than the kernel ahead, moe_wide_mid_kernel; the first: ids,
    // which say what groups of few slots there are)
    int expert = 0, slots = 0, groups = -1;
    bool waited = false;
    if (!OUT && p.slots <= 32) {
        const Few few(p);
        if (few.fit) {
            groups = few.groups();
            uint32_t of = 0u;
            if ((int)blockIdx.y < groups) few.group(blockIdx.y, expert, of);
            slots = __popc(of);
        }
    }
    if (groups < 0) {
        if (!OUT) {
            grid_dependency_wait();
            grid_launch_dependents();
            waited = true;
        }
        const uint4 first = load_16(p.w.group + blockIdx.y);   // (what is there of a group that is not is not used)
        groups = *p.w.groups;
        expert = (int)first.x;
        slots = (int)first.y;
    }
    for (int i = blockIdx.y; i < groups; i += gridDim.y) {
        if (i != (int)blockIdx.y) {
            expert = p.w.group[i].expert;
            slots = p.w.group[i].n;
        }
        Wide<OUT, XT, GP> w(p, p.w.group + i, expert, slots, smem);
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s) w.issue();
        if (!waited) {
            grid_dependency_wait();
            grid_launch_dependents();
            waited = true;
        }
        if (OUT) {
            // (as many words ahead as there are registers for)
            if (slots <= 4) w.template run_out<1, 4>();
            else if (MOST == 1) w.template run_out<2, 2>();
            else if (slots <= 8) w.template run_out<2, 4>();
            else if (slots <= 12) w.template run_out<3, 2>();
            else w.template run_out<4, 2>();
        } else {
            if (MOST == 1 || slots <= 8) w.template run_in<1>();
            else w.template run_in<2>();
        }
    }
    if (!waited) {
        grid_dependency_wait();
        grid_launch_dependents();
    }
}

// y = residual + what a token's slots add, in their order; eight columns a thread
template <class T> __global__ void __launch_bounds__(128) moe_combine_kernel(const __grid_constant__ MoeParams p)
{
    const int t = blockIdx.y, c = (blockIdx.x * 128 + threadIdx.x) * 8;
    grid_dependency_wait();
    grid_launch_dependents();
    if (c >= p.H) return;
    float v[8] = {};
    if (p.residual) dsq_unpack8(dsq_load8((const T *)p.residual + (int64_t)t * p.H + c), v);
    for (int s = 0; s < p.k; ++s) {
        const int id = p.ids[t * p.k + s];
        if (id < 0 || id >= p.E) continue;
        const float4 *from = reinterpret_cast<const float4 *>(p.w.part + (int64_t)(t * p.k + s) * p.H + c);
        const float4 a = from[0], b = from[1];
        v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
        v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
    }
    DsqRaw8<T> r;
    dsq_pack8(v, r);
    dsq_store8((T *)p.Y + (int64_t)t * p.H + c, r);
}

// ---- host
template <bool OUT, int XT, int GP, int MOST> int launch(const MoeParams &p, cudaStream_t s)
{
    constexpr int bytes = Wide<OUT, XT, GP>::BYTES, cols = WC * (OUT ? 32 : 16);
    static_assert(bytes <= 112 * 1024, "shared memory");
    static std::atomic<unsigned long long> configured{0};
    const auto kernel = moe_wide_kernel<OUT, XT, GP, MOST>;
    const int st = dsq_allow_smem((const void *)kernel, bytes, &configured);
    if (st) return st;
    // (of mid to the end of the last chunk: zeros)
    const int columns = OUT ? p.H : p.chunks_out * 128;
    const dim3 grid((unsigned)((columns + cols - 1) / cols), (unsigned)p.groups_most());
    return dsq_launch(kernel, grid, dim3(THREADS), (size_t)bytes, s, dsq_launch_hooks().pdl, 0, p);
}
template <bool OUT, int XT> int pick(const MoeParams &p, int gp, cudaStream_t s)
{
    if (p.rows == 8)
        return gp == 4 ? launch<OUT, XT, 4, 1>(p, s) : gp == 2 ? launch<OUT, XT, 2, 1>(p, s) : launch<OUT, XT, 1, 1>(p, s);
    return gp == 4 ? launch<OUT, XT, 4, 2>(p, s) : gp == 2 ? launch<OUT, XT, 2, 2>(p, s) : launch<OUT, XT, 1, 2>(p, s);
}
template <class T> int combine(const MoeParams &p, cudaStream_t s)
{
    return dsq_launch(moe_combine_kernel<T>, dim3((unsigned)((p.H + 1023) / 1024), (unsigned)p.T), dim3(128), 0, s,
                      dsq_launch_hooks().pdl, 0, p);
}

}  // namespace

int dsq_moe::run_wide(const MoeParams &p, int x_type, int gp_in, int gp_out, cudaStream_t s)
{
    const int pdl = dsq_launch_hooks().pdl;
    int st;
    if (p.scaled)
        st = dsq_launch(gp_in == 4 ? moe_wide_prepare_scaled_kernel<true> : moe_wide_prepare_scaled_kernel<false>, dim3(1 + p.T), dim3(256),
                        0, s, pdl, 0, p);
    else
        st = dsq_launch(gp_in == 4 ? moe_wide_prepare_kernel<true> : moe_wide_prepare_kernel<false>,
                        dim3(1 + (p.T * p.chunks_in + PREPARE_WARPS - 1) / PREPARE_WARPS), dim3(PREPARE_WARPS * 32), 0, s, pdl, 0, p);
    if (!st) st = x_type == DSQ_BF16 && !p.scaled ? pick<false, DSQ_BF16>(p, gp_in, s) : pick<false, DSQ_F16>(p, gp_in, s);
    if (!st) st = dsq_launch(gp_out == 4 ? moe_wide_mid_kernel<true> : moe_wide_mid_kernel<false>, dim3(p.slots), dim3(256), 0, s, pdl, 0, p);
    if (!st) st = pick<true, DSQ_F16>(p, gp_out, s);
    if (!st)
        st = p.y_type == DSQ_F32 ? combine<float>(p, s) : p.y_type == DSQ_BF16 ? combine<__nv_bfloat16>(p, s) : combine<__half>(p, s);
    return st;
}
