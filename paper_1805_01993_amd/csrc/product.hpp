// Matrix products of a block on the matrix cores: what a launch is given.  C[m][n] = sum over k of M[m][k] N[n][k].
#pragma once

#include "element.hpp"

namespace ccdc {

// One side of a product, in 16-bit numbers: rows of k, or (strided) rows of that side's index with k from row to row.  Rows begin on
// 16 bytes and are whole packs of them; what is past a row's end in its last pack is zero.
struct Side {
    const uint16_t *p;
    int64_t ld;                   // elements between rows
    int64_t plane;                // elements between the planes of an fp32 side
    int64_t segment;              // elements from the first range of k to the second
    int32_t columns;              // strided: elements of a row that may be read, a multiple of 8
};

enum class Product {
    gated,                        // N: W_in, M: x.  h (and what the backward needs) from a and u
    plain,                        // N: W_out, M: h.  y
    parts,                        // the same in ranges of k, a product each, in fp32: what k_parts adds up
    gated_gradient,               // N: W_out strided, M: dy.  gradients of a and u from that of h
    input_gradient,               // N: W_in strided, M: gradients of a and u.  dx
    weight_gradient               // both strided, a product per file: dW_in, dW_out
};

struct ProductArgs {
    Side n, m;
    int32_t rows_n, rows_m;       // of the result; gated: rows_n is the hidden size
    int32_t K, segments;          // weight_gradient: the files' tokens on average, for the choice of a tile
    int32_t tiles_n, tiles_m;
    const int32_t *first;         // weight_gradient: rows of k where the files begin
    int32_t part_k;               // parts: k of a range, whole steps; files is their number
    int32_t files, halves;        // halves: products a file has, side M of the second from its segment on
    void *c;                      // result
    int64_t ldc, file_c, half_c;
    // gated, gated_gradient: matrices of the hidden values
    uint16_t *h;                  // gated: h; gated_gradient: gradient of a, of u from h_second on
    int64_t ldh, plane_h, second_h;
    float *P, *Q;                 // gradient of h to those of a and u, [rows_m][ldh], P -0 where both are 0; gated: null: not wanted
    const RowOf *row_of;
    Dropout drop;
    int32_t activation;
};

// Launches a product of the mode (ccdc_mode); chooses the tile.
int run_product(int mode, Product what, ProductArgs a, hipStream_t st);

// What follows a product is in kernels of several tiles, of which one file's values may come from one and on another node from another:
// with the same operations in each, none that the compiler has put together (a product and a sum in one rounding) in one of them only.
#define CCDC_AS_WRITTEN _Pragma("clang fp contract(off)")

// The three bfloat16 numbers of an fp32 number.  Rounded to nearest, so that what is left is at most 2^-9 of it; near the
// largest numbers, where that would be an infinity, cut instead.  Infinities and NaN are their first part.
__device__ __forceinline__ void split(float x, uint16_t *part)
{
    CCDC_AS_WRITTEN
    float first = HybBF16::widen(narrow<ElemBF16>(x));
    if (fabsf(first) > 3.4e38f) first = __uint_as_float(__float_as_uint(x) & 0xFFFF0000u);
    const float left = fabsf(first) <= 3.4e38f ? x - first : 0.0f;
    part[0] = (uint16_t)(__float_as_uint(first) >> 16);
    part[1] = narrow<ElemBF16>(left);
    part[2] = narrow<ElemBF16>(left - HybBF16::widen(part[1]));
}

// Eight numbers as a side of a later product.
template <class T>
__device__ __forceinline__ void store_side(uint16_t *p, int64_t plane, const Eight &x)
{
    using P = Pack<uint16_t, 8>;
    if constexpr (T::planes == 1) {
        store_eight<T>(p, x, 8);
    } else {
        P q[3];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            uint16_t part[3];
            split(x.v[i], part);
            q[0].v[i] = part[0], q[1].v[i] = part[1], q[2].v[i] = part[2];
        }
#pragma unroll
        for (int s = 0; s < 3; s++) *reinterpret_cast<P *>(p + s * plane) = q[s];
    }
}

// The activation of a and its derivative.  16-bit modes: the hardware's exponential of x, some |x| 2^-24 of its value off, which the
// rounding of h to 8 or 11 bits hides (8192 rows of 4096 x 11264 bf16 1919 us, with expf 1945).
template <class T>
__device__ __forceinline__ void activate(int which, float a, float &value, float &slope)
{
    CCDC_AS_WRITTEN
    if (which == CCDC_ACT_SILU) {
        const float e = T::planes == 1 ? __expf(-a) : expf(-a), s = 1.0f / (1.0f + e);
        value = a * s;
        slope = s * fmaf(a, 1.0f - s, 1.0f);
    } else if (which == CCDC_ACT_GELU) {
        const float cdf = 0.5f * (1.0f + erff(a * 0.70710678f));
        value = a * cdf;
        slope = fmaf(a * 0.39894228f, T::planes == 1 ? __expf(-0.5f * a * a) : expf(-0.5f * a * a), cdf);
    } else {
        value = a > 0.0f ? a : a != a ? a : 0.0f;
        slope = a > 0.0f ? 1.0f : 0.0f;
    }
}

// The forward for at most kFewRows rows (few.hip).
constexpr int64_t kFewRows = 64;
int few_forward(const ccdc_block_t *b, int64_t rows, const void *x, int64_t ldx, const void *W_in, const void *W_out, void *y, int64_t ldy,
                void *h, const Dropout &drop, hipStream_t st);

// The bytes of a workspace or of what is saved from `at` on.
template <class E = void>
inline E *inside_of(const void *base, size_t at)
{
    return reinterpret_cast<E *>(const_cast<char *>(static_cast<const char *>(base)) + at);
}

}  // namespace ccdc
