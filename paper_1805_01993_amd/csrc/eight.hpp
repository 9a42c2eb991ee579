// Matrices in 8 bits (ccdc.h): rows of e4m3 numbers in whole blocks of 128, each with a power of two.
#pragma once

#include "element.hpp"

namespace ccdc {

constexpr int64_t kMostColumns = (int64_t)1 << 20;      // of a row of the calls that learn from a teacher

// Bytes of a row, and of its scales.
constexpr int64_t packed_columns(int64_t columns) { return (columns + 127) / 128 * 128; }
constexpr int64_t packed_scales(int64_t columns) { return (packed_columns(columns) / 128 + 3) / 4 * 4; }

// What a product of two such matrices is given.  C[m][n] = sum over k of M[m][k] N[n][k].
struct Product8Args {
    const uint8_t *n, *m, *n_scale, *m_scale;
    int32_t ld, ld_scale;         // bytes of a row, and of its scales
    int32_t rows_n, rows_m, blocks;
    int32_t tiles_n, tiles_m;
    void *c;
    int64_t ldc;
};

typedef int Bytes32 __attribute__((ext_vector_type(8)));      // 32 numbers of a row
typedef int Bytes16 __attribute__((ext_vector_type(4)));
typedef __bf16 Wide2 __attribute__((ext_vector_type(2)));
typedef __bf16 Wide8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ Bytes32 both(Bytes16 low, Bytes16 high)
{
    return __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7);
}

// 2^(scale - 127).  (0 stands for 2^-127, which is no normal number.)
__device__ __forceinline__ float power(int scale)
{
    return __int_as_float(scale > 0 ? scale << 23 : 1 << 22);
}

// Eight numbers of 8 bits times a power of two, as bfloat16: exact where the scale leaves them in its range (below).
__device__ __forceinline__ Wide8 wide(int low, int high, float scale)
{
    const Wide2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, scale, true);
    const Wide2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, scale, true);
    return Wide8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// fp32 results: the numbers as bfloat16 with their scale, whose products the instructions add in fp32 (ccdc.h has what they drop in 8 bits,
// 2^-14 or so of a result).
//
// All numbers of 8 bits (2^-9 to 1.75 2^8) times 2^(scale - 127) are normal bfloat16 numbers, 2^-126 to less than 2^128, for scales of
// 10 to 246.  A wavefront that has seen another one, in any block, makes its sums once more, from memory, with scales handed over as below:
// blocks next to the ends of fp32's range, which a block of the other side may bring back.  Apart from the loop, because all that a wavefront
// has in registers there leaves none for a second way: within it the kernels of tiles took 157 to 185 registers for 118.
constexpr int kLowestScale = 10, kHighestScale = 246;
struct ScalesSeen {
    uint32_t most = 0;
    __device__ __forceinline__ void see(int scale) { most = max(most, (uint32_t)(scale - kLowestScale)); }
    __device__ __forceinline__ bool others() const { return __any(most > (uint32_t)(kHighestScale - kLowestScale)); }
};

// One side hands the other 2^16: the product of two scales is what it was, and each is within.  (What is so far out that the other has no
// room for it has a product past fp32's range, and still has when it takes what room there is.)  255 is no number and stays it.  Rows
// are of three kinds, within, above and below, so the products are added in five turns, each of the rows that have the same to hand over and
// of zeros in place of the others: what a pair of rows gets is the same whatever rows are beside it.
//   turn          0 within, within   1 above, any   2 below, any   3 within, above   4 within, below
//   n's scale     as it is           / 2^16         2^16           2^16              / 2^16
constexpr int kScaleTurns = 5;
struct ScaleInTurn {
    int scale, mask;                      // mask: 0 where the row has another turn
};
__device__ __forceinline__ ScaleInTurn scale_in_turn(int scale, bool of_n, int turn)
{
    const int kind = scale == 255 ? 0 : scale > kHighestScale ? 1 : scale < kLowestScale ? 2 : 0, own = turn > 2 ? turn - 2 : turn;
    const int handed = turn == 0 ? 0 : (turn == 1 || turn == 4) == of_n ? -16 : 16;
    const bool in = turn == 0 ? kind == 0 : turn <= 2 ? !of_n || kind == own : kind == (of_n ? 0 : own);
    return {scale == 255 ? 255 : min(max(scale + handed, kLowestScale), kHighestScale), in ? -1 : 0};
}
__device__ __forceinline__ Wide8 wide_in_turn(int low, int high, ScaleInTurn s)
{
    Bytes16 bits = __builtin_bit_cast(Bytes16, wide(low, high, power(s.scale)));
#pragma unroll
    for (int i = 0; i < 4; i++) bits[i] &= s.mask;
    return __builtin_bit_cast(Wide8, bits);
}

// The products of a few rows (few8.hip), where they are the faster, and of more (product8.hip).
bool few_rows8(const ccdc_block_t *b, const Product8Args &a);
int few_product8(const ccdc_block_t *b, const Product8Args &a, hipStream_t st);
int tiled_product8(const ccdc_block_t *b, const Product8Args &a, hipStream_t st);

}  // namespace ccdc
