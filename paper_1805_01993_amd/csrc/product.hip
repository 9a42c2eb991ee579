// Matrix products of a block: C[m][n] = sum over k of M[m][k] N[n][k], with what follows the product done on the result in
// registers.
//
// A workgroup makes a tile of C: its wavefronts 32 x 32 pieces of it by v_mfma_f32_32x32x16, rows of N as the
// instruction's rows, so that a lane ends with runs of four n of one m (eight after an exchange between the wavefront's
// halves: a whole pack of a row of C, and the eight columns that one call of dropout's generator decides on).  Steps of
// 64 k of both sides are copied into LDS past the registers, the next step while this one is computed on.
//
// A side whose k is contiguous lies in LDS as [row][64 k], one that is strided as [64 k][row]; the latter's pieces are
// read with the transposing LDS read.  Both lie in an order that spreads what a wavefront reads together over
// the banks; the copy writes LDS lane by lane, so it is the lanes' global addresses that are permuted.
//
// fp32: every number is the sum of three bfloat16 numbers (24 bits of mantissa in three times 8), and the product the
// sum of the six products of them that are not below 2^-24 of it, small ones first.  Six 16-bit products are 2.7 times
// the rate of one in fp32 on these matrix cores.
//
// Every element of C is one chain of sums over k in steps of 16, whatever the tile: its bits depend on its row and column alone.
#include "product.hpp"

#ifndef CCDC_PRODUCT_PART
#define CCDC_PRODUCT_PART 0
#endif

namespace {
using namespace ccdc;

typedef float Acc __attribute__((ext_vector_type(16)));
typedef short Bits4 __attribute__((ext_vector_type(4)));
typedef short Bits8 __attribute__((ext_vector_type(8)));
typedef __bf16 Bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 Half8 __attribute__((ext_vector_type(8)));
#define CCDC_LDS __attribute__((address_space(3)))

constexpr int kStep = 64;         // k of a step

__device__ const uint32_t zeros[4] = {};       // what is read in place of k past the end

template <class T>
__device__ __forceinline__ Acc multiply(Bits8 n, Bits8 m, Acc c)
{
    if constexpr (std::is_same<T, ElemF16>::value)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(Half8, n), __builtin_bit_cast(Half8, m), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(Bf8, n), __builtin_bit_cast(Bf8, m), c, 0, 0, 0);
}

// Copies 16 bytes a lane to LDS, lane after lane from byte `to` on.  The compiler does not count these: every step's are
// waited for in one place.
__device__ __forceinline__ void copy_to_lds(uint32_t to, const void *base, uint32_t offset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :: "s"(to), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ void copy_to_lds(uint32_t to, const void *from)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(to), "v"(from) : "memory");
}

// Bytes in LDS of pack `pack` (eight k) of row `row`, k contiguous: the eight rows that are read together are in different banks.
__device__ __forceinline__ uint32_t contiguous_at(uint32_t row, uint32_t pack) { return row * 128 + ((pack ^ (row & 7)) * 16); }
// Place in its row of pack `pack` (eight rows of the side) at k, strided: the four k that are read together, 32 rows of
// the side each, are in different banks.
__device__ __forceinline__ uint32_t strided_pack(uint32_t k, uint32_t pack) { return pack ^ ((k & 3) << 2); }

// The copies of one side that a wavefront makes in each step.
template <bool STRIDED, int ROWS, int THREADS>
struct Copies {
    static constexpr int count = ROWS * 8 / THREADS;
    const uint16_t *base[count];          // the same for all lanes
    uint32_t offset[count];               // bytes, a lane's own
    uint32_t to;                          // byte in LDS of the first

    // GATED: rows r of a tile are 32 of Wg and 32 of Wu in turn.
    template <bool GATED>
    __device__ __forceinline__ void set(const Side &s, int32_t row0, int32_t rows, uint32_t lds)
    {
        const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
        to = lds + wave * 1024;
#pragma unroll
        for (int i = 0; i < count; i++) {
            const uint32_t p = i * THREADS + wave * 64;       // the first lane's pack
            if constexpr (STRIDED) {
                constexpr uint32_t packs = ROWS / 8;
                const uint32_t k = (p + lane) / packs, pack = strided_pack(k, (p + lane) % packs);
                const int32_t column = min(row0 + (int32_t)pack * 8, s.columns - 8) - row0;
                base[i] = s.p + row0;
                offset[i] = (uint32_t)((k * s.ld + column) * 2);
            } else {
                int32_t r = p / 8, second = 0;
                if constexpr (GATED) {
                    second = r / 32 % 2;
                    r = r / 64 * 32 + r % 32;
                }
                const int32_t from = min(row0 + r, rows - 1);
                const uint32_t row = p / 8 + lane / 8;        // in LDS
                const int32_t at = min(from + (int32_t)(lane / 8), rows - 1) - from;
                base[i] = s.p + (from + (int64_t)second * rows) * s.ld;
                offset[i] = (uint32_t)((at * s.ld + ((lane % 8) ^ (row & 7)) * 8) * 2);
            }
        }
    }
    // k0 .. k0 + 63 from element `from` of the side on; left: how many of them there are.
    __device__ __forceinline__ void issue(const Side &s, int64_t from, int32_t k0, int32_t left, uint32_t buffer) const
    {
        from += STRIDED ? k0 * s.ld : k0;
#pragma unroll
        for (int i = 0; i < count; i++) {
            const uint16_t *b = base[i] + from;
            const uint32_t at = __builtin_amdgcn_readfirstlane(to + buffer + i * THREADS * 16);
            if (left >= kStep) {
                copy_to_lds(at, b, offset[i]);
            } else {
                const uint32_t lane = threadIdx.x % 64, p = i * THREADS + threadIdx.x / 64 * 64 + lane;
                const int32_t k = STRIDED ? p / (ROWS / 8) : ((lane % 8) ^ ((p / 8) & 7)) * 8;
                const void *q = (const char *)b + offset[i];
                copy_to_lds(at, k < left ? q : zeros);
            }
        }
    }
};

// The piece of 32 rows from row0 on and 16 k from k0 on, as the matrix instruction takes it: lane l row l % 32, k 8 (l / 32) ...
template <bool STRIDED, int ROWS>
__device__ __forceinline__ Bits8 piece(CCDC_LDS unsigned char *lds, int row0, int k0)
{
    const uint32_t lane = threadIdx.x % 64;
    if constexpr (STRIDED) {
        // four k of sixteen rows by each group of sixteen lanes; a lane's address is of four rows at one k
        const uint32_t k = k0 + lane / 32 * 8 + lane % 16 / 4, row = row0 + lane / 16 % 2 * 16 + lane % 4 * 4;
        CCDC_LDS unsigned char *p = lds + k * (ROWS * 2) + strided_pack(k, row / 8) * 16 + row % 8 * 2;
        const Bits4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((CCDC_LDS Bits4 *)p);
        const Bits4 high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((CCDC_LDS Bits4 *)(p + 4 * ROWS * 2));
        return __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
        return *(CCDC_LDS Bits8 *)(lds + contiguous_at(row0 + lane % 32, k0 / 8 + lane / 32));
    }
}

// Eight n of one m: n 16 half + 8 (lane / 32) ... of the piece, after the wavefront's halves have exchanged runs of four.
__device__ __forceinline__ Eight eight_of(const Acc &c, int half)
{
    Eight out;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(c[8 * half + k]), __float_as_uint(c[8 * half + 4 + k]), false, false);
        out.v[k] = __uint_as_float(r[0]);
        out.v[4 + k] = __uint_as_float(r[1]);
    }
    return out;
}

// The activation of a and its derivative.
template <class T>
__device__ __forceinline__ void activate(int which, float a, float &value, float &slope)
{
    if (which == CCDC_ACT_SILU) {
        const float e = T::planes == 1 ? __expf(-a) : expf(-a), s = 1.0f / (1.0f + e);
        value = a * s;
        slope = s * (1.0f + a * (1.0f - s));
    } else if (which == CCDC_ACT_GELU) {
        const float cdf = 0.5f * (1.0f + erff(a * 0.70710678f));
        value = a * cdf;
        slope = cdf + a * 0.39894228f * (T::planes == 1 ? __expf(-0.5f * a * a) : expf(-0.5f * a * a));
    } else {
        value = a > 0.0f ? a : a != a ? a : 0.0f;
        slope = a > 0.0f ? 1.0f : 0.0f;
    }
}

// WN x WM wavefronts, each SN x SM pieces.
template <class T, Product WHAT, int WN, int WM, int SN, int SM>
__global__ __launch_bounds__(64 * WN * WM) void k_product(const ProductArgs a)
{
    constexpr bool NS = WHAT != Product::gated && WHAT != Product::plain, MS = WHAT == Product::weight_gradient;
    constexpr bool GATED = WHAT == Product::gated;
    constexpr int THREADS = 64 * WN * WM, TN = WN * SN * 32, TM = WM * SM * 32, BUFFER = (TN + TM) * kStep * 2;
    __shared__ __attribute__((aligned(1024))) unsigned char memory[2 * BUFFER];
    CCDC_LDS unsigned char *lds = (CCDC_LDS unsigned char *)memory;
    const uint32_t lds_at = (uint32_t)(uintptr_t)lds;

    // Tiles: an XCD takes a contiguous range of them, in groups of eight rows of tiles, so that what its workgroups
    // read at one time is a few rows of tiles of either side.
    constexpr uint32_t kGroup = 8;
    const uint32_t block = xcd_contiguous(blockIdx.x, gridDim.x), per = a.tiles_n * a.tiles_m;
    const uint32_t product = block / per, t = block - product * per, in_group = kGroup * a.tiles_n;
    const uint32_t group = t / in_group, rows_in = min(a.tiles_m - group * kGroup, kGroup), in = t - group * in_group;
    const int32_t tile_m = (group * kGroup + in % rows_in) * TM, tile_n = in / rows_in * (GATED ? TN / 2 : TN);

    Side sn = a.n, sm = a.m;
    int32_t K = a.K, file = 0, half = 0;
    if constexpr (WHAT == Product::weight_gradient) {
        file = product / a.halves;
        half = product - file * a.halves;
        const int32_t from = a.first[file];
        K = a.first[file + 1] - from;
        sn.p += from * sn.ld;
        sm.p += from * sm.ld + half * sm.segment;
    }
    Copies<NS, TN, THREADS> cn;
    Copies<MS, TM, THREADS> cm;
    cn.template set<GATED>(sn, tile_n, a.rows_n, lds_at);
    cm.template set<false>(sm, tile_m, a.rows_m, lds_at + TN * kStep * 2);

    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int wn = wave % WN * SN * 32, wm = wave / WN * SM * 32;
    Acc acc[SN][SM];
#pragma unroll
    for (int i = 0; i < SN; i++)
#pragma unroll
        for (int j = 0; j < SM; j++)
#pragma unroll
            for (int e = 0; e < 16; e++) acc[i][j][e] = 0.0f;

    // steps: planes of either side, then ranges of k, then k
    const int32_t in_k = (K + kStep - 1) / kStep, steps = in_k * a.segments * (T::planes == 1 ? 1 : 6);
    int32_t next_k = 0, next_segment = 0, next_planes = 0;
    const auto issue = [&](uint32_t buffer) {
        int64_t from_n = next_segment ? sn.segment : 0, from_m = next_segment ? sm.segment : 0;
        if constexpr (T::planes == 3) {           // (2,0) (0,2) (1,1) (1,0) (0,1) (0,0)
            const int pn = (0x001102 >> (4 * next_planes)) & 15, pm = (0x010120 >> (4 * next_planes)) & 15;
            from_n += pn * sn.plane;
            from_m += pm * sm.plane;
        }
        const int32_t k0 = next_k * kStep, left = K - k0;
        cn.issue(sn, from_n, k0, left, buffer);
        cm.issue(sm, from_m, k0, left, buffer);
        if (++next_k == in_k) {
            next_k = 0;
            if (++next_segment == a.segments) next_segment = 0, next_planes++;
        }
    };

    if (steps > 0) issue(0);
    for (int32_t s = 0; s < steps; s++) {
        // this step's copies are there, and every wavefront has read the step before it
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (s + 1 < steps) issue((s + 1) % 2 * BUFFER);
        CCDC_LDS unsigned char *n = lds + s % 2 * BUFFER, *m = n + TN * kStep * 2;
#pragma unroll
        for (int k = 0; k < kStep; k += 16) {
            Bits8 pn[SN], pm[SM];
#pragma unroll
            for (int i = 0; i < SN; i++) pn[i] = piece<NS, TN>(n, wn + i * 32, k);
#pragma unroll
            for (int j = 0; j < SM; j++) pm[j] = piece<MS, TM>(m, wm + j * 32, k);
#pragma unroll
            for (int i = 0; i < SN; i++)
#pragma unroll
                for (int j = 0; j < SM; j++) acc[i][j] = multiply<T>(pn[i], pm[j], acc[i][j]);
        }
    }

#pragma unroll
    for (int j = 0; j < SM; j++) {
        const int32_t m = tile_m + wm + j * 32 + lane % 32;
        const bool row_there = m < a.rows_m;
        RowOf of{};
        if (GATED && a.drop.threshold && row_there) of = a.row_of[m];
#pragma unroll
        for (int half_n = 0; half_n < 2; half_n++) {
            if constexpr (GATED) {
                static_assert(!GATED || SN == 2);
                const int32_t f = tile_n + wn / 2 + half_n * 16 + lane / 32 * 8;
                const Eight va = eight_of(acc[0][j], half_n), vu = eight_of(acc[1][j], half_n);
                if (!row_there || f >= a.ldh) continue;
                Eight h, P, Q, keep;
                if (a.drop.threshold) keep = dropout_factors(a.drop, of.id, of.token, f / 8);
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    float value, slope;
                    activate<T>(a.activation, va.v[e], value, slope);
                    h.v[e] = value * vu.v[e], P.v[e] = slope * vu.v[e], Q.v[e] = value;
                    if (a.drop.threshold) h.v[e] = kept(h.v[e], keep.v[e]), P.v[e] = kept(P.v[e], keep.v[e]), Q.v[e] = kept(Q.v[e], keep.v[e]);
                    if (f + e >= a.rows_n) h.v[e] = P.v[e] = Q.v[e] = 0.0f;
                }
                const int64_t at = (int64_t)m * a.ldh + f;
                store_side<T>(a.h + at, a.plane_h, h);
                if (a.P) {
                    store_eight<ElemF32>(a.P + at, P, 8);
                    store_eight<ElemF32>(a.Q + at, Q, 8);
                }
            } else {
#pragma unroll
                for (int i = 0; i < SN; i++) {
                    const int32_t n = tile_n + wn + i * 32 + half_n * 16 + lane / 32 * 8;
                    Eight v = eight_of(acc[i][j], half_n);
                    if constexpr (WHAT == Product::gated_gradient) {
                        if (!row_there || n >= a.ldh) continue;
                        const int64_t at = (int64_t)m * a.ldh + n;
                        const Eight P = load_eight<ElemF32>(a.P + at, 8), Q = load_eight<ElemF32>(a.Q + at, 8);
                        Eight da, du;
#pragma unroll
                        for (int e = 0; e < 8; e++) {
                            da.v[e] = v.v[e] * P.v[e], du.v[e] = v.v[e] * Q.v[e];
                            if (n + e >= a.rows_n) da.v[e] = du.v[e] = 0.0f;
                        }
                        uint16_t *to = a.h + (int64_t)m * 2 * a.ldh + n;
                        store_side<T>(to, a.plane_h, da);
                        store_side<T>(to + a.second_h, a.plane_h, du);
                    } else {
                        if (!row_there || n >= a.rows_n) continue;
                        typename T::elem *to = (typename T::elem *)a.c + file * a.file_c + half * a.half_c + (int64_t)m * a.ldc + n;
                        store_eight<T>(to, v, a.rows_n - n);
                    }
                }
            }
        }
    }
}

template <class T, Product WHAT, int WN, int WM, int SN, int SM>
int launch(ProductArgs a, hipStream_t st)
{
    a.tiles_n = cdiv(a.rows_n, WN * SN * 32 / (WHAT == Product::gated ? 2 : 1));
    a.tiles_m = cdiv(a.rows_m, WM * SM * 32);
    const uint64_t tiles = (uint64_t)a.tiles_n * a.tiles_m * a.files * a.halves;
    if (!fits_launch(tiles * 64 * WN * WM)) return CCDC_ESIZE;
    k_product<T, WHAT, WN, WM, SN, SM><<<(uint32_t)tiles, 64 * WN * WM, 0, st>>>(a);
    return launched();
}

// 256 x 256 tiles where they fill the chip.
template <class T, Product WHAT>
int by_tile(const ProductArgs &a, hipStream_t st)
{
    const uint64_t large = (uint64_t)cdiv(a.rows_n, WHAT == Product::gated ? 128 : 256) * cdiv(a.rows_m, 256) * a.files * a.halves;
    if (large >= 256) return launch<T, WHAT, 4, 2, 2, 4>(a, st);
    return launch<T, WHAT, 2, 2, 2, 2>(a, st);
}

template <class T>
int by_product(Product what, const ProductArgs &a, hipStream_t st)
{
    switch (what) {
    case Product::gated: return by_tile<T, Product::gated>(a, st);
    case Product::plain: return by_tile<T, Product::plain>(a, st);
    case Product::gated_gradient: return by_tile<T, Product::gated_gradient>(a, st);
    case Product::input_gradient: return by_tile<T, Product::input_gradient>(a, st);
    default: return by_tile<T, Product::weight_gradient>(a, st);
    }
}

}  // namespace

namespace ccdc {

// One element type a compilation.
int run_product_f32(Product what, const ProductArgs &a, hipStream_t st);
int run_product_bf16(Product what, const ProductArgs &a, hipStream_t st);
int run_product_f16(Product what, const ProductArgs &a, hipStream_t st);
#if CCDC_PRODUCT_PART == 0
int run_product_f32(Product what, const ProductArgs &a, hipStream_t st) { return by_product<ElemF32>(what, a, st); }

int run_product(int mode, Product what, ProductArgs a, hipStream_t st)
{
    if (a.rows_n <= 0 || a.rows_m <= 0 || a.files <= 0) return CCDC_OK;
    switch (mode) {
    case CCDC_BF16_SUM_XOR: return run_product_bf16(what, a, st);
    case CCDC_F16_SUM_XOR: return run_product_f16(what, a, st);
    default: return run_product_f32(what, a, st);
    }
}
#elif CCDC_PRODUCT_PART == 1
int run_product_bf16(Product what, const ProductArgs &a, hipStream_t st) { return by_product<ElemBF16>(what, a, st); }
#else
int run_product_f16(Product what, const ProductArgs &a, hipStream_t st) { return by_product<ElemF16>(what, a, st); }
#endif

}  // namespace ccdc
