// Products of a few rows in 8 bits: an answer's next tokens.  The time is that of reading the weights once, a byte each, so they go from
// memory to the matrix instructions' registers without a stop in LDS.
//
// As in few.hip a wavefront multiplies 16 x 16 pieces, here by v_mfma_scale_f32_16x16x128: 16 / S rows of the weights in S parts
// of their k, and as many rows of x in the same parts; only the products of equal parts are wanted.  A part of a step is a whole
// block of 128, so each of the instruction's rows has one scale, which the instruction applies.  Its lanes have 32 of a row's 128
// numbers, any 32, the same ones on both sides.
#include "eight.hpp"

namespace {
using namespace ccdc;

typedef float Acc4 __attribute__((ext_vector_type(4)));

struct Block8 {
    Bytes32 q;
    int scale;
};

__device__ __forceinline__ Block8 load_block(const uint8_t *q, const uint8_t *scale, int32_t block)
{
    const uint8_t *p = q + (int64_t)block * 128;
    return {both(*(const Bytes16 *)p, *(const Bytes16 *)(p + 64)), scale[block]};
}

// fp32 results: the numbers as bfloat16 with their scale, whose products the instructions add in fp32 (ccdc.h has what they drop in
// 8 bits, 2^-14 or so of a result).
template <class T>
__device__ __forceinline__ Acc4 multiply(const Block8 &n, const Block8 &m, Acc4 c)
{
    if constexpr (T::planes == 1) {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(n.q, m.q, c, 0, 0, 0, n.scale, 0, m.scale);
    } else {
        const float sn = power(n.scale), sm = power(m.scale);
#pragma unroll
        for (int i = 0; i < 4; i++)
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide(n.q[2 * i], n.q[2 * i + 1], sn), wide(m.q[2 * i], m.q[2 * i + 1], sm), c, 0, 0, 0);
        return c;
    }
}

template <class T, int S, int MT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_few8(const Product8Args a)
{
    using E = typename T::elem;
    constexpr int R = 16 / S, COLUMNS = MT * R, AHEAD = MT > 4 ? 1 : MT > 1 ? 2 : 4;
    __shared__ float sums[WAVES][MT][16][17];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane % 16, part = r % S;
    const int32_t n0 = blockIdx.x * R;
    const int64_t row_n = min(n0 + r / S, a.rows_n - 1);
    const uint8_t *w = a.n + row_n * a.ld + lane / 16 * 16, *w_scale = a.n_scale + row_n * a.ld_scale;
    const uint8_t *x[MT], *x_scale[MT];
#pragma unroll
    for (int t = 0; t < MT; t++) {
        const int64_t row = min(t * R + r / S, a.rows_m - 1);
        x[t] = a.m + row * a.ld + lane / 16 * 16;
        x_scale[t] = a.m_scale + row * a.ld_scale;
    }
    Acc4 acc[MT] = {};
    const int32_t steps = (a.blocks + S - 1) / S;
    for (int32_t s = wave; s < steps; s += AHEAD * WAVES) {
        Block8 bw[AHEAD], bx[AHEAD][MT];
#pragma unroll
        for (int u = 0; u < AHEAD; u++) {
            const int32_t block = min((s + u * WAVES) * S + part, a.blocks - 1);      // past the end: not added
            bw[u] = load_block(w, w_scale, block);
#pragma unroll
            for (int t = 0; t < MT; t++) bx[u][t] = load_block(x[t], x_scale[t], block);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; u++) {
            if (s + u * WAVES >= steps) continue;
            // the step that the row ends in: zeros on both sides, and scales of one (a block that is no number stays out)
            if ((s + u * WAVES + 1) * S > a.blocks) {
                const int in = (s + u * WAVES) * S + part < a.blocks ? -1 : 0;
                const auto keep = [in](Block8 &b) {
#pragma unroll
                    for (int i = 0; i < 8; i++) b.q[i] &= in;
                    b.scale = in ? b.scale : 127;
                };
                keep(bw[u]);
#pragma unroll
                for (int t = 0; t < MT; t++) keep(bx[u][t]);
            }
#pragma unroll
            for (int t = 0; t < MT; t++) acc[t] = multiply<T>(bw[u], bx[u][t], acc[t]);
        }
    }
    // lane l has rows 4 (l / 16) ... of column l % 16
#pragma unroll
    for (int t = 0; t < MT; t++)
#pragma unroll
        for (int e = 0; e < 4; e++) sums[wave][t][lane / 16 * 4 + e][r] = acc[t][e];
    __syncthreads();
    for (int o = threadIdx.x; o < R * COLUMNS; o += 64 * WAVES) {
        const int n = o % R, c = o / R;
        if (n0 + n >= a.rows_n || c >= a.rows_m) continue;
        float total = 0.0f;
#pragma unroll
        for (int v = 0; v < WAVES; v++)
#pragma unroll
            for (int p = 0; p < S; p++) total += sums[v][c * S / 16][n * S + p][c * S % 16 + p];
        ((E *)a.c)[c * a.ldc + n0 + n] = narrow<T>(total);
    }
}

template <class T>
int run_few8(const Product8Args &a, hipStream_t st)
{
    const auto go = [&](auto s, auto mt, auto waves) -> int {
        constexpr int S = decltype(s)::value, MT = decltype(mt)::value, WAVES = decltype(waves)::value;
        const uint32_t blocks = cdiv(a.rows_n, 16 / S);
        if (!fits_launch((uint64_t)blocks * 64 * WAVES)) return CCDC_ESIZE;
        k_few8<T, S, MT, WAVES><<<blocks, 64 * WAVES, 0, st>>>(a);
        return launched();
    };
    using std::integral_constant;
    if (a.rows_m <= 4) return go(integral_constant<int, 4>(), integral_constant<int, 1>(), integral_constant<int, 4>());
    if (a.rows_m <= 8) return go(integral_constant<int, 2>(), integral_constant<int, 1>(), integral_constant<int, 4>());
    if (a.rows_m <= 16) return go(integral_constant<int, 1>(), integral_constant<int, 1>(), integral_constant<int, 8>());
    if (a.rows_m <= 32) return go(integral_constant<int, 1>(), integral_constant<int, 2>(), integral_constant<int, 8>());
    return go(integral_constant<int, 1>(), integral_constant<int, 4>(), integral_constant<int, 8>());
}

}  // namespace

namespace ccdc {

int few_product8(const ccdc_block_t *b, const Product8Args &a, hipStream_t st) { CCDC_BY_ELEM(b, (run_few8<T>(a, st))); }

}  // namespace ccdc
