// The feed-forward block for a few rows: an answer's next tokens.  The time is that of reading the weights once, so they go from
// memory to the matrix instructions' registers without a stop in LDS, as many loads in flight as the chip has room for.
//
// h is rounded to the block's elements between the two products, as in product.hip.
//
// A wavefront multiplies 16 x 16 pieces by v_mfma_f32_16x16x32, rows of the weights as the instruction's rows.  Its 16 rows are 16 / S
// rows of the weights in S parts of their k, and its 16 columns as many rows of x in the same S parts: the products of equal
// parts are what is wanted, the others come for nothing.  With few rows of x that makes a workgroup's share of the weights
// 16 / S rows, so there are S times the workgroups, and a row's loads are S times as long: one row of x, 2048 x 4160 bf16, is
// 1040 and 512 workgroups (8.0 and 5.5 us: 4.3 and 3.1 TB/s).  Two parts also make whole lines of a load's rows: with up to 16 rows of x, then two
// pieces of columns, 12.4 -> 8.8 and 8.7 -> 6.4 us, with 64 in eight 24.6 -> 19.8 and 25.4 -> 12.7; four parts with more than four rows were
// slower again (x is read more often).  A workgroup's wavefronts take steps of 32 S k in turn; their sums are added in LDS in
// the wavefronts' order.  More steps on their way than AHEAD took the registers of a second workgroup.
#include "product.hpp"

namespace {
using namespace ccdc;

typedef float Acc4 __attribute__((ext_vector_type(4)));
typedef short Raw8 __attribute__((ext_vector_type(8)));
typedef __bf16 Bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 Half8 __attribute__((ext_vector_type(8)));

// Eight k of a row, as the instruction takes them (fp32: three parts).
template <class T>
struct Operand {
    Raw8 part[T::planes];
};

// As loaded.
template <class T>
struct Loaded {
    Pack<typename T::elem, 16 / sizeof(typename T::elem)> p[sizeof(typename T::elem) / 2];
};

template <class T>
__device__ __forceinline__ Loaded<T> load_k(const typename T::elem *p)
{
    using P = Pack<typename T::elem, 16 / sizeof(typename T::elem)>;
    Loaded<T> v;
#pragma unroll
    for (int h = 0; h < (int)sizeof(typename T::elem) / 2; h++)
        v.p[h] = load_pack_any<true, P, typename T::elem>(p + h * (16 / sizeof(typename T::elem)));
    return v;
}

// The same where a row may end: zeros past it.
template <class T>
__device__ __forceinline__ Loaded<T> load_end(const typename T::elem *p, int left)
{
    constexpr int W = 16 / sizeof(typename T::elem);
    left = fresh(left);
    if (left >= 8) return load_k<T>(p);
    Loaded<T> v;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const typename T::elem e = p[min(i, left - 1)];      // the row's last element where it has ended
        if constexpr (T::planes == 1) v.p[i / W].v[i % W] = (uint16_t)(e & -inside(left, i));
        else v.p[i / W].v[i % W] = __int_as_float(__float_as_int(e) & -inside(left, i));
    }
    return v;
}

template <class T>
__device__ __forceinline__ Operand<T> operand(const Loaded<T> &v)
{
    Operand<T> o;
    if constexpr (T::planes == 1) {
        o.part[0] = __builtin_bit_cast(Raw8, v.p[0]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            uint16_t part[3];
            split(v.p[i / 4].v[i % 4], part);
#pragma unroll
            for (int s = 0; s < 3; s++) o.part[s][i] = (short)part[s];
        }
    }
    return o;
}

template <class T>
__device__ __forceinline__ Acc4 multiply(const Operand<T> &n, const Operand<T> &m, Acc4 c)
{
    const auto one = [&](int i, int j) {
        if constexpr (std::is_same<T, ElemF16>::value)
            c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(Half8, n.part[i]), __builtin_bit_cast(Half8, m.part[j]), c, 0, 0, 0);
        else
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Bf8, n.part[i]), __builtin_bit_cast(Bf8, m.part[j]), c, 0, 0, 0);
    };
    if constexpr (T::planes == 3) one(2, 0), one(0, 2), one(1, 1), one(1, 0), one(0, 1);
    one(0, 0);
    return c;
}

struct FewArgs {
    const void *w, *x;
    void *y;
    int64_t ldw, ldx, ldy;
    int32_t rows_n, rows_m, K;
    const RowOf *row_of;
    Dropout drop;
    int32_t activation;
};

// GATED: y is h = D(act(a) u), a and u by rows n and rows_n + n of w.
template <class T, bool GATED, int S, int MT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_few(const FewArgs a)
{
    using E = typename T::elem;
    constexpr int R = 16 / S, STREAMS = GATED ? 2 : 1, STEP = 32 * S, COLUMNS = MT * 16 / S, AHEAD = T::planes == 3 ? (MT > 2 ? 1 : 2) : MT > 4 ? 1 : MT > 1 ? 2 : 4;
    __shared__ float sums[WAVES][STREAMS][MT][16][17];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane % 16;
    const int32_t n0 = blockIdx.x * R, offset = r % S * 32 + lane / 16 * 8;
    const E *w[STREAMS], *x[MT];
#pragma unroll
    for (int i = 0; i < STREAMS; i++)
        w[i] = (const E *)a.w + ((int64_t)min(n0 + r / S, a.rows_n - 1) + (i ? a.rows_n : 0)) * a.ldw + offset;
#pragma unroll
    for (int t = 0; t < MT; t++) x[t] = (const E *)a.x + (int64_t)min(t * R + r / S, a.rows_m - 1) * a.ldx + offset;

    Acc4 acc[STREAMS][MT] = {};
    const int32_t whole = a.K / STEP;
    const auto add = [&](const Loaded<T> (&lw)[STREAMS], const Loaded<T> (&lx)[MT]) {
        Operand<T> ox[MT];
#pragma unroll
        for (int t = 0; t < MT; t++) ox[t] = operand<T>(lx[t]);
#pragma unroll
        for (int i = 0; i < STREAMS; i++) {
            const Operand<T> ow = operand<T>(lw[i]);
#pragma unroll
            for (int t = 0; t < MT; t++) acc[i][t] = multiply<T>(ow, ox[t], acc[i][t]);
        }
    };
    // The step that the rows end in is one wavefront's, asked for before its whole ones and added after them.
    const bool last = a.K % STEP && whole % WAVES == wave;
    Loaded<T> ew[STREAMS], ex[MT];
    if (last) {
        const int64_t k = (int64_t)whole * STEP;
        const int left = a.K - (int)k - offset;
#pragma unroll
        for (int i = 0; i < STREAMS; i++) ew[i] = load_end<T>(w[i] + k, left);
#pragma unroll
        for (int t = 0; t < MT; t++) ex[t] = load_end<T>(x[t] + k, left);
    }
    for (int32_t s = wave; s < whole; s += AHEAD * WAVES) {
        Loaded<T> lw[AHEAD][STREAMS], lx[AHEAD][MT];
#pragma unroll
        for (int u = 0; u < AHEAD; u++) {
            const int64_t k = (int64_t)min(s + u * WAVES, whole - 1) * STEP;      // past the wavefront's steps: not added
#pragma unroll
            for (int i = 0; i < STREAMS; i++) lw[u][i] = load_k<T>(w[i] + k);
#pragma unroll
            for (int t = 0; t < MT; t++) lx[u][t] = load_k<T>(x[t] + k);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; u++)
            if (s + u * WAVES < whole) add(lw[u], lx[u]);
    }
    if (last) add(ew, ex);

    // lane l has rows 4 (l / 16) ... of column l % 16
#pragma unroll
    for (int i = 0; i < STREAMS; i++)
#pragma unroll
        for (int t = 0; t < MT; t++)
#pragma unroll
            for (int e = 0; e < 4; e++) sums[wave][i][t][lane / 16 * 4 + e][r] = acc[i][t][e];
    __syncthreads();
    for (int o = threadIdx.x; o < R * COLUMNS; o += 64 * WAVES) {
        const int n = o % R, c = o / R;
        const int32_t column = n0 + n;
        if (column >= a.rows_n || c >= a.rows_m) continue;
        float total[STREAMS];
#pragma unroll
        for (int i = 0; i < STREAMS; i++) {
            total[i] = 0.0f;
#pragma unroll
            for (int v = 0; v < WAVES; v++)
#pragma unroll
                for (int p = 0; p < S; p++) total[i] += sums[v][i][c * S / 16][n * S + p][c * S % 16 + p];
        }
        float result = total[0];
        if constexpr (GATED) {
            float value, slope;
            activate<T>(a.activation, total[0], value, slope);
            result = value * total[1];
            if (a.drop.threshold) {
                const RowOf of = a.row_of[c];
                const Eight f = dropout_factors(a.drop, of.id, of.token, column / 8);
                float factor = f.v[0];
#pragma unroll
                for (int e = 1; e < 8; e++) factor = column % 8 == e ? f.v[e] : factor;
                result = kept(result, factor);
            }
        }
        ((E *)a.y)[c * a.ldy + column] = narrow<T>(result);
    }
}

template <class T, bool GATED>
int run_few(const FewArgs &a, hipStream_t st)
{
    const auto go = [&](auto s, auto mt, auto waves) {
        constexpr int S = decltype(s)::value, MT = decltype(mt)::value, WAVES = decltype(waves)::value;
        k_few<T, GATED, S, MT, WAVES><<<cdiv(a.rows_n, 16 / S), 64 * WAVES, 0, st>>>(a);
        return launched();
    };
    using std::integral_constant;
    constexpr bool wide = T::planes == 3;         // three times the registers an operand: no parts for more than sixteen rows
    if (a.rows_m <= 4) return go(integral_constant<int, 4>(), integral_constant<int, 1>(), integral_constant<int, GATED ? 4 : 8>());
    if (a.rows_m <= 8) return go(integral_constant<int, 2>(), integral_constant<int, 1>(), integral_constant<int, 8>());
    if (a.rows_m <= 16) return go(integral_constant<int, 2>(), integral_constant<int, 2>(), integral_constant<int, GATED ? 8 : 16>());
    if (a.rows_m <= 32)
        return go(integral_constant<int, wide ? 1 : 2>(), integral_constant<int, wide ? 2 : 4>(),
                  integral_constant<int, !GATED ? 16 : wide ? 8 : 4>());
    return go(integral_constant<int, wide ? 1 : 2>(), integral_constant<int, wide ? 4 : 8>(), integral_constant<int, GATED && !wide ? 4 : 8>());
}

}  // namespace

namespace ccdc {

// h is a matrix of the block's elements in this form.
int few_forward(const ccdc_block_t *b, int64_t rows, const void *x, int64_t ldx, const void *W_in, const void *W_out, void *y, int64_t ldy,
                void *h, const Dropout &drop, hipStream_t st)
{
    const int64_t d = b->c.width, F = b->c.hidden;
    const FewArgs in{W_in, x, h, d, ldx, b->hidden_ld, (int32_t)F, (int32_t)rows, (int32_t)d, b->d_row_of, drop, b->c.activation};
    const FewArgs out{W_out, h, y, F, b->hidden_ld, ldy, (int32_t)d, (int32_t)rows, (int32_t)F, b->d_row_of, {}, 0};
    const auto gated = [&]() -> int { CCDC_BY_ELEM(b, (run_few<T, true>(in, st))); };
    const auto plain = [&]() -> int { CCDC_BY_ELEM(b, (run_few<T, false>(out, st))); };
    const int rc = gated();
    return rc == CCDC_OK ? plain() : rc;
}

}  // namespace ccdc
