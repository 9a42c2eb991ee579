// Products of a few rows in 8 bits: an answer's next tokens.  The time is that of reading the weights once, a byte each, so they go from
// memory to the matrix instructions' registers without a stop in LDS.
//
// As in few.hip a wavefront multiplies 16 x 16 pieces, here by v_mfma_scale_f32_16x16x128: 16 / S rows of the weights in S parts
// of their k, and as many rows of x in the same parts; only the products of equal parts are wanted.  What is multiplied at a time is a
// whole block of 128, so each of the instruction's rows has one scale, which the instruction applies.  Its lanes have 32 of a row's
// 128 numbers, any 32, the same ones on both sides.
//
// x comes from L2 as often as there are groups of rows of the weights, and costs there what the weights do, so a workgroup has G
// groups where that leaves enough workgroups; and scales are read a word of four at a time, or they are a third of the loads.  One row, 4096 x
// 11264 (46 MB): one group, a scale at a time 14.8 us, two groups 11.1, and words 10.7 (4.3 TB/s; a kernel that does nothing takes 2).
// From 9 rows on LDS's copies are worth their way where the weights have many rows (16 rows of 4096 x 11264: 15.3 us here, 14.6 by
// tiles of 64 x 64; of 1600 x 32768 15.3, 12.4; of 11264 x 4096 13.7, 32).  With fp32 results rows go by here up to 32 and,
// of few outputs, 64 (4096 x 11264, 16 rows 13.9 us, tiles 21.9; 32 rows 21.1, 22.1; 64 of 11264 x 4096 23.0, 55; but 24 of 1600 x 32768 21.0, 13.5).
// Loads of a next step begun before this one's products lost more by those past the rows' ends than they gave (14.8 us).
// Of few outputs there are fewer workgroups than CUs, and more than 16 rows are divided among workgroups too: a group of 8 or 16 outputs
// for 8, 16 or 32 rows, whichever leaves a CU the least to read.  64 rows of 11264 x 1024 12.2 us by 16 x 16 (16 x 32 18.2, 8 x 8 22.4, tiles of
// 64 x 64 31.5), x 2048 19.3 by 16 x 32 (32.0 by tiles), x 4096 25.0 by 32 x 32 (34.0), x 6000 34.6 by tiles (45.4); 16 rows of 11264 x
// 1024 7.2 by 8 x 8, 12.1 by 16 x 16.
#include <algorithm>

#include "eight.hpp"

namespace {
using namespace ccdc;

typedef float Acc4 __attribute__((ext_vector_type(4)));

struct Block8 {
    Bytes32 q;
    int scale;                            // in its lowest byte
};

template <class T>
__device__ __forceinline__ Acc4 multiply(const Block8 &n, const Block8 &m, Acc4 c)
{
    if constexpr (T::planes == 1) {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(n.q, m.q, c, 0, 0, 0, n.scale, 0, m.scale);
    } else {
        const float sn = power(n.scale & 255), sm = power(m.scale & 255);
#pragma unroll
        for (int i = 0; i < 4; i++)
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide(n.q[2 * i], n.q[2 * i + 1], sn), wide(m.q[2 * i], m.q[2 * i + 1], sm), c, 0, 0, 0);
        return c;
    }
}

// The same where scales leave bfloat16's range.
__device__ __forceinline__ Acc4 multiply_in_turns(const Block8 &n, const Block8 &m, Acc4 c)
{
#pragma unroll 1
    for (int turn = 0; turn < kScaleTurns; turn++) {
        const ScaleInTurn sn = scale_in_turn(n.scale, true, turn), sm = scale_in_turn(m.scale, false, turn);
#pragma unroll
        for (int i = 0; i < 4; i++)
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide_in_turn(n.q[2 * i], n.q[2 * i + 1], sn), wide_in_turn(m.q[2 * i], m.q[2 * i + 1], sm), c, 0, 0, 0);
    }
    return c;
}

// One row's share of a lane: its numbers and scales.
struct Line {
    const uint8_t *q, *scale;
    __device__ __forceinline__ void set(const uint8_t *base, const uint8_t *scales, int64_t row, const Product8Args &a)
    {
        q = base + row * a.ld + threadIdx.x % 64 / 16 * 16;
        scale = scales + row * a.ld_scale;
    }
    // One block by itself; past the end as k_few8 has it.
    __device__ __forceinline__ Block8 block(int32_t b, const Product8Args &a) const
    {
        const uint8_t *p = q + (int64_t)min(b, a.blocks - 1) * 128;
        Block8 o{both(*(const Bytes16 *)p, *(const Bytes16 *)(p + 64)), scale[min(b, a.blocks - 1)]};
        if (b >= a.blocks) o = {Bytes32{}, 127};
        return o;
    }
};

// NB blocks of a line from a multiple of NB on, as loaded: their scales are one word.
template <int NB>
struct Batch {
    Bytes16 q[NB][2];
    uint32_t scales;
    __device__ __forceinline__ void load(const Line &l, const int32_t (&block)[NB], int32_t word)
    {
#pragma unroll
        for (int b = 0; b < NB; b++) {
            const uint8_t *p = l.q + (int64_t)block[b] * 128;
            q[b][0] = *(const Bytes16 *)p;
            q[b][1] = *(const Bytes16 *)(p + 64);
        }
        scales = *(const uint32_t *)(l.scale + word);
    }
    __device__ __forceinline__ Block8 of(int b, int shift) const { return {both(q[b][0], q[b][1]), (int)(scales >> (shift + 8 * b))}; }
};

// G groups of 16 / S rows of the weights a workgroup.  Part p of a row is its blocks p B ..., B a multiple of four; a wavefront takes NB of
// them at a time, in turns with the others.
template <class T, int S, int MT, int WAVES, int G, int NB>
__global__ __launch_bounds__(64 * WAVES) void k_few8(const Product8Args a)
{
    using E = typename T::elem;
    constexpr int R = 16 / S, COLUMNS = MT * R;
    __shared__ float sums[WAVES][G][MT][16][17];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane % 16, part = r % S;
    const int32_t n0 = blockIdx.x * (R * G), m0 = blockIdx.y * COLUMNS, B = ((a.blocks + S - 1) / S + 3) / 4 * 4, first = part * B;
    Line w[G], x[MT];
#pragma unroll
    for (int g = 0; g < G; g++) w[g].set(a.n, a.n_scale, min(n0 + g * R + r / S, a.rows_n - 1), a);
#pragma unroll
    for (int t = 0; t < MT; t++) x[t].set(a.m, a.m_scale, min(m0 + t * R + r / S, a.rows_m - 1), a);
    Acc4 acc[G][MT] = {};
    ScalesSeen seen;
    for (int32_t s = wave * NB; s < B; s += WAVES * NB) {
        int32_t block[NB];
#pragma unroll
        for (int b = 0; b < NB; b++) block[b] = min(first + s + b, a.blocks - 1);     // past the end: not added
        Batch<NB> bw[G], bx[MT];
        const int32_t word = block[0] / 4 * 4;
#pragma unroll
        for (int g = 0; g < G; g++) bw[g].load(w[g], block, word);
#pragma unroll
        for (int t = 0; t < MT; t++) bx[t].load(x[t], block, word);
        const int shift = s % 4 * 8;
        const bool ends = (S - 1) * B + s + NB > a.blocks;            // for some lane
#pragma unroll
        for (int b = 0; b < NB; b++) {
            Block8 ow[G], ox[MT];
#pragma unroll
            for (int g = 0; g < G; g++) ow[g] = bw[g].of(b, shift);
#pragma unroll
            for (int t = 0; t < MT; t++) ox[t] = bx[t].of(b, shift);
            if (ends) {
                // past the end: zeros on both sides, and scales of one (a block that is no number stays out)
                const int in = first + s + b < a.blocks ? -1 : 0;
                const auto keep = [in](Block8 &o) {
#pragma unroll
                    for (int i = 0; i < 8; i++) o.q[i] &= in;
                    o.scale = in ? o.scale : 127;
                };
#pragma unroll
                for (int g = 0; g < G; g++) keep(ow[g]);
#pragma unroll
                for (int t = 0; t < MT; t++) keep(ox[t]);
            }
            if constexpr (T::planes == 3) {
#pragma unroll
                for (int g = 0; g < G; g++) seen.see(ow[g].scale & 255);
#pragma unroll
                for (int t = 0; t < MT; t++) seen.see(ox[t].scale & 255);
            }
#pragma unroll
            for (int g = 0; g < G; g++)
#pragma unroll
                for (int t = 0; t < MT; t++) acc[g][t] = multiply<T>(ow[g], ox[t], acc[g][t]);
        }
    }
    if constexpr (T::planes == 3)
        if (seen.others()) {
#pragma unroll
            for (int g = 0; g < G; g++)
#pragma unroll
                for (int t = 0; t < MT; t++) {
                    Acc4 sum = {};
#pragma unroll 1
                    for (int32_t s = wave * NB; s < B; s += WAVES * NB)
#pragma unroll 1
                        for (int b = 0; b < NB; b++) sum = multiply_in_turns(w[g].block(first + s + b, a), x[t].block(first + s + b, a), sum);
                    acc[g][t] = sum;
                }
        }
    // lane l has rows 4 (l / 16) ... of column l % 16
#pragma unroll
    for (int g = 0; g < G; g++)
#pragma unroll
        for (int t = 0; t < MT; t++)
#pragma unroll
            for (int e = 0; e < 4; e++) sums[wave][g][t][lane / 16 * 4 + e][r] = acc[g][t][e];
    __syncthreads();
    for (int o = threadIdx.x; o < R * G * COLUMNS; o += 64 * WAVES) {
        const int n = o % (R * G), c = o / (R * G), in = n % R;
        if (n0 + n >= a.rows_n || m0 + c >= a.rows_m) continue;
        float total = 0.0f;
#pragma unroll
        for (int v = 0; v < WAVES; v++)
#pragma unroll
            for (int p = 0; p < S; p++) total += sums[v][n / R][c * S / 16][in * S + p][c * S % 16 + p];
        ((E *)a.c)[(m0 + c) * a.ldc + n0 + n] = narrow<T>(total);
    }
}

template <class T>
int run_few8(const Product8Args &a, hipStream_t st)
{
    const auto go = [&](auto s, auto mt, auto waves, auto g, auto nb) -> int {
        constexpr int S = decltype(s)::value, MT = decltype(mt)::value, WAVES = decltype(waves)::value, G = decltype(g)::value, NB = decltype(nb)::value;
        const uint32_t blocks = cdiv(a.rows_n, 16 / S * G), rows = cdiv(a.rows_m, 16 / S * MT);
        if (!fits_launch((uint64_t)blocks * rows * 64 * WAVES)) return CCDC_ESIZE;
        k_few8<T, S, MT, WAVES, G, NB><<<dim3(blocks, rows), 64 * WAVES, 0, st>>>(a);
        return launched();
    };
    using std::integral_constant;
    const integral_constant<int, 1> one;
    const integral_constant<int, 2> two;
    const integral_constant<int, 4> four;
    const integral_constant<int, 8> eight;
    const bool wide = a.rows_n >= 8192;               // with two groups a workgroup there still are enough workgroups
    if (a.rows_m <= 4 && a.rows_n < 2048) return go(four, one, four, one, two);
    if (a.rows_m <= 8) return wide ? go(two, one, eight, two, two) : go(two, one, eight, one, two);
    if constexpr (T::planes == 3)                     // (16-bit results go by tiles there)
        if (wide) return a.rows_m <= 16 ? go(one, one, four, four, two) : go(one, two, eight, two, two);
    // the fewest rows, of both sides, that a CU has to read (what it takes from L2 or memory is some 45 GB/s)
    const auto read = [&](uint32_t n, uint32_t m) { return cdiv((uint64_t)cdiv(a.rows_n, n) * cdiv(a.rows_m, m), 256) * (n + m); };
    const auto small = read(8, 8), square = read(16, 16), tall = read(16, 32), large = read(32, 32), least = std::min(std::min(small, square), std::min(tall, large));
    if (square == least) return go(one, one, eight, one, two);
    if (small == least) return go(two, one, eight, one, two);
    return tall == least ? go(one, two, eight, one, two) : go(one, two, eight, two, two);
}

}  // namespace

namespace ccdc {

bool few_rows8(const ccdc_block_t *b, const Product8Args &a)
{
    if (a.rows_m > 64 || a.blocks < 8) return false;
    if (a.rows_m <= 8) return true;
    if (a.rows_m <= 32) return a.rows_n < 8192 || b->planes == 3;
    return a.rows_n <= 4096;
}

int few_product8(const ccdc_block_t *b, const Product8Args &a, hipStream_t st) { CCDC_BY_ELEM(b, (run_few8<T>(a, st))); }

}  // namespace ccdc
