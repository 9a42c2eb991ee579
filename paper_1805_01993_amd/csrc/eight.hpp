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

// Eight numbers of 8 bits times a power of two, as bfloat16: exact.
__device__ __forceinline__ Wide8 wide(int low, int high, float scale)
{
    const Wide2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, scale, true);
    const Wide2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, scale, true);
    return Wide8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The products of a few rows (few8.hip), where they are the faster, and of more (product8.hip).
bool few_rows8(const ccdc_block_t *b, const Product8Args &a);
int few_product8(const ccdc_block_t *b, const Product8Args &a, hipStream_t st);
int tiled_product8(const ccdc_block_t *b, const Product8Args &a, hipStream_t st);

}  // namespace ccdc
