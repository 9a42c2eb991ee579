// Matrices in 8 bits: how they are made, and the entry of their product.
#include "eight.hpp"

namespace {
using namespace ccdc;

struct QuantiseArgs {
    const void *x;
    uint8_t *q, *scale;
    int64_t ldx;
    int32_t columns, ld, ld_scale;
    uint32_t packs, rows;             // eight columns each, of a row; whole blocks
};

// The largest of sixteen lanes, in all of them.
__device__ __forceinline__ uint32_t most_of_16(uint32_t v)
{
    const auto moved = [](uint32_t x, auto control) {
        return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(control)::value, 15, 15, true);
    };
    using std::integral_constant;
    v = max(v, moved(v, integral_constant<int, 0x121>()));          // rotated by 1, 2, 4 and 8 lanes
    v = max(v, moved(v, integral_constant<int, 0x122>()));
    v = max(v, moved(v, integral_constant<int, 0x124>()));
    return max(v, moved(v, integral_constant<int, 0x128>()));
}

// A lane has eight numbers of a row, sixteen lanes a block.  The scale is a power of two: numbers are divided by it without a rounding, so
// that e4m3's alone is left (at most 2^-4 of the number from 2^-6 of the scale on), and the matrix instructions take it as it is.
// Against the largest number over 448 that leaves up to one of the four bits of exponent unused.
template <class T>
__global__ __launch_bounds__(kBlock) void k_quantise(const QuantiseArgs a)
{
    const uint64_t p = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
    const uint32_t row = (uint32_t)(p / a.packs), pack = (uint32_t)(p - (uint64_t)row * a.packs);
    if (row >= a.rows) return;                    // (whole blocks of lanes: packs is a multiple of sixteen)
    const int c = (int)pack * 8;
    Eight v = {};
    if (c < a.columns) v = load_eight<T>((const typename T::elem *)a.x + row * a.ldx + c, a.columns - c);
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const uint32_t bits = __float_as_uint(v.v[i]) & 0x7FFFFFFFu;
        most = max(most, bits < 0x7F800000u ? bits : 0u);
    }
    most = most_of_16(most);
    // 448 = 1.75 2^8
    int e = (int)(most >> 23) - 127 - 8 + ((most & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    e = most == 0 ? 0 : max(e, -127);
    typedef int Two __attribute__((ext_vector_type(2)));
    Two out;
#pragma unroll
    for (int h = 0; h < 2; h++) {
        float s[4];
#pragma unroll
        for (int i = 0; i < 4; i++) s[i] = ldexpf(v.v[h * 4 + i], -e);
        const int low = __builtin_amdgcn_cvt_pk_fp8_f32(s[0], s[1], 0, false);
        out[h] = __builtin_amdgcn_cvt_pk_fp8_f32(s[2], s[3], low, true);
    }
    *(Two *)(a.q + (int64_t)row * a.ld + c) = out;
    if (pack % 16 == 0) {
        uint8_t *scale = a.scale + (int64_t)row * a.ld_scale;
        const int block = (int)pack / 16, blocks = (int)a.packs / 16;
        scale[block] = (uint8_t)(e + 127);
        if (block == blocks - 1)
            for (int b = blocks; b < a.ld_scale; b++) scale[b] = 127;
    }
}

template <class T>
int run_quantise(const QuantiseArgs &a, hipStream_t st)
{
    k_quantise<T><<<cdiv((uint64_t)a.rows * a.packs, kBlock), kBlock, 0, st>>>(a);
    return launched();
}

}  // namespace

extern "C" {

int ccdc_quantise(const ccdc_block_t *b, int64_t rows, int64_t columns, const void *x, int64_t ldx, void *q, void *scale, void *stream)
{
    const int rc = ready(b);
    if (rc != CCDC_OK) return rc;
    if (rows < 0 || columns < 1 || ldx < columns) return CCDC_EINVAL;
    if (rows == 0) return CCDC_OK;
    if (!fits(b, x) || !q || !scale || !aligned(q, 16) || !aligned(scale, 4)) return CCDC_EINVAL;
    if (columns > kMostColumns || rows > INT32_MAX) return CCDC_ESIZE;
    const int32_t ld = (int32_t)packed_columns(columns);
    if (!fits_launch((uint64_t)rows * (ld / 8) + kBlock)) return CCDC_ESIZE;
    const QuantiseArgs a{x, (uint8_t *)q, (uint8_t *)scale, ldx, (int32_t)columns, ld, (int32_t)packed_scales(columns), (uint32_t)ld / 8,
                         (uint32_t)rows};
    CCDC_BY_ELEM(b, (run_quantise<T>(a, (hipStream_t)stream)));
}

int ccdc_packed_product(const ccdc_block_t *b, int64_t rows, int64_t outputs, int64_t columns, const void *x, const void *x_scale, const void *W,
                  const void *W_scale, void *y, int64_t ldy, void *stream)
{
    const int rc = ready(b);
    if (rc != CCDC_OK) return rc;
    if (rows < 0 || outputs < 1 || columns < 1 || ldy < outputs) return CCDC_EINVAL;
    if (rows == 0) return CCDC_OK;
    for (const void *p : {x, W})
        if (!p || !aligned(p, 16)) return CCDC_EINVAL;
    for (const void *p : {x_scale, W_scale})
        if (!p || !aligned(p, 4)) return CCDC_EINVAL;
    if (!fits(b, y)) return CCDC_EINVAL;
    if (columns > kMostColumns || rows > INT32_MAX || outputs > INT32_MAX) return CCDC_ESIZE;
    const int32_t ld = (int32_t)packed_columns(columns);
    const Product8Args a{(const uint8_t *)W, (const uint8_t *)x, (const uint8_t *)W_scale, (const uint8_t *)x_scale, ld,
                         (int32_t)packed_scales(columns), (int32_t)outputs, (int32_t)rows, ld / 128, 0, 0, y, ldy};
    return few_rows8(b, a) ? few_product8(b, a, (hipStream_t)stream) : tiled_product8(b, a, (hipStream_t)stream);
}

}  // extern "C"
