// Matrix products of a block: C[m][n] = sum over k of M[m][k] N[n][k], with what follows the product done on the result in
// registers.
//
// A workgroup makes a tile of C: its wavefronts 32 x 32 pieces of it by v_mfma_f32_32x32x16, rows of N as the
// instruction's rows.  Steps of 64 k of both sides (fp32: 32 k of three parts) are copied into LDS past the registers while
// those before are computed on.  Large tiles (256 x 256, eight wavefronts, 128 KB of LDS) where they fill the chip, else 128 x 128.
// Bound by the matrix cores and the copies to LDS beside them, at the card's power limit: 8192 x 4096 x 11264 bf16 1.17
// PFLOP/s (643 us; the products alone, nothing read or copied, 505), 14336 x 8320 x 2048 with what follows it 0.77.
//
// A side whose k is contiguous lies in LDS as [row][64 k], one that is strided as [64 k][row]; the latter's pieces are
// read with the transposing LDS read.  Both lie in an order that spreads what a wavefront reads together over
// the banks (without it a read took twice as long); the copy writes LDS lane by lane, so it is the lanes' global addresses
// that are permuted.
//
// fp32: every number is the sum of three bfloat16 numbers (24 bits of mantissa in three times 8), and the product the
// sum of the six products of them that are not below 2^-24 of it.  Six 16-bit products are 2.7 times the rate of one in
// fp32 on these matrix cores.
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


__device__ const uint32_t zeros[4] = {};       // what is read in place of k past the end

// P of a hidden value that dropout took out.
constexpr float kTakenOut = -0.0f;

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

// Place in its row of pack `pack` (eight k) of row `row`, k contiguous, `packs` of them a row: sixteen rows are read together, and the
// banks hold 16 / packs of them beside one another, so each so many rows have an order of their own.
template <uint32_t packs>
__device__ __forceinline__ uint32_t contiguous_pack(uint32_t row, uint32_t pack) { return pack ^ (row / (16 / packs) % packs); }
// Place in its row of pack `pack` (eight rows of the side) at k, strided: the four k that are read together, 32 rows of
// the side each, are in different banks.
__device__ __forceinline__ uint32_t strided_pack(uint32_t k, uint32_t pack) { return pack ^ ((k & 3) << 2); }

// The copies of one side that a wavefront makes in each step of STEP k.
template <bool STRIDED, int ROWS, int THREADS, int STEP>
struct Copies {
    static constexpr bool strided = STRIDED;
    static constexpr int count = ROWS * (STEP / 8) / THREADS;
    static constexpr uint32_t packs = STRIDED ? ROWS / 8 : STEP / 8;      // of a row in LDS
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
                const uint32_t k = (p + lane) / packs, pack = strided_pack(k, (p + lane) % packs);
                const int32_t column = min(row0 + (int32_t)pack * 8, s.columns - 8) - row0;
                base[i] = s.p + row0;
                offset[i] = (uint32_t)((k * s.ld + column) * 2);
            } else {
                int32_t r = p / packs, second = 0;
                if constexpr (GATED) {
                    second = r / 32 % 2;
                    r = r / 64 * 32 + r % 32;
                }
                const int32_t from = min(row0 + r, rows - 1);
                const uint32_t row = (p + lane) / packs;      // in LDS
                const int32_t at = min(from + (int32_t)(lane / packs), rows - 1) - from;
                base[i] = s.p + (from + (int64_t)second * rows) * s.ld;
                offset[i] = (uint32_t)((at * s.ld + contiguous_pack<packs>(row, lane % packs) * 8) * 2);
            }
        }
    }
    // Copy i of the k from element `from` of the side on, of which there are `left`.
    __device__ __forceinline__ void issue(int i, int64_t from, int32_t left, uint32_t buffer) const
    {
        const uint16_t *b = base[i] + from;
        const uint32_t at = __builtin_amdgcn_readfirstlane(to + buffer + i * THREADS * 16);
        if (left >= STEP) {
            copy_to_lds(at, b, offset[i]);
        } else {
            const uint32_t lane = threadIdx.x % 64, p = i * THREADS + threadIdx.x / 64 * 64 + lane;
            const int32_t k = STRIDED ? p / packs : contiguous_pack<STEP / 8>(p / packs, lane % packs) * 8;
            const void *q = (const char *)b + offset[i];
            copy_to_lds(at, k < left ? q : zeros);
        }
    }
};

// The piece of 32 rows from row0 on and 16 k from k0 on, as the matrix instruction takes it: lane l row l % 32, k 8 (l / 32) ...
template <bool STRIDED, int ROWS, int STEP>
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
        const uint32_t row = row0 + lane % 32;
        return *(CCDC_LDS Bits8 *)(lds + row * (STEP * 2) + contiguous_pack<STEP / 8>(row, k0 / 8 + lane / 32) * 16);
    }
}

// WN x WM wavefronts, each SN x SM pieces; BUFFERS steps in LDS.
template <class T, Product WHAT, int WN, int WM, int SN, int SM, int BUFFERS>
__global__ __launch_bounds__(64 * WN * WM) void k_product(const ProductArgs a)
{
    constexpr bool NS = WHAT != Product::gated && WHAT != Product::plain && WHAT != Product::parts, MS = WHAT == Product::weight_gradient;
    constexpr bool GATED = WHAT == Product::gated;
    constexpr int THREADS = 64 * WN * WM, TN = WN * SN * 32, TM = WM * SM * 32;
    // fp32: a step has all planes of 32 k, so that each is copied and read once for the products that it is in
    // (small tiles of gradients of weights: files are often shorter than 64 tokens, and with half the LDS a CU has three of them)
    constexpr int PLANES = T::planes, STEP = PLANES == 3 || (WHAT == Product::weight_gradient && SM == 1) ? 32 : 64, PLANE = (TN + TM) * STEP * 2, BUFFER = PLANES * PLANE;
    __shared__ __attribute__((aligned(1024))) unsigned char memory[BUFFERS * BUFFER];
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
    if constexpr (WHAT == Product::parts) {
        file = product;
        const int64_t from = (int64_t)file * a.part_k;
        K = (int32_t)min(a.K - from, (int64_t)a.part_k);
        sn.p += from;
        sm.p += from;
    }
    Copies<NS, TN, THREADS, STEP> cn;
    Copies<MS, TM, THREADS, STEP> cm;
    cn.template set<GATED>(sn, tile_n, a.rows_n, lds_at);
    cm.template set<false>(sm, tile_m, a.rows_m, lds_at + TN * STEP * 2);

    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int wn = wave % WN * SN * 32, wm = wave / WN * SM * 32;
    Acc acc[SN][SM];
#pragma unroll
    for (int i = 0; i < SN; i++)
#pragma unroll
        for (int j = 0; j < SM; j++)
#pragma unroll
            for (int e = 0; e < 16; e++) acc[i][j][e] = 0.0f;

    // steps: k, then ranges of k; each has all planes of either side
    const int32_t in_k = (K + STEP - 1) / STEP, steps = in_k * a.segments;
    // What is copied next of a side: its place in the side's order of steps.
    struct Next {
        int32_t k = 0, segment = 0;
    };
    Next next_n, next_m;
    const auto copies = [&](const auto &side, const Side &s, Next &at, uint32_t buffer) {
        constexpr bool strided = std::decay_t<decltype(side)>::strided;
        const int64_t k0 = (int64_t)at.k * STEP, from = (at.segment ? s.segment : 0) + (strided ? k0 * s.ld : k0);
#pragma unroll
        for (int plane = 0; plane < PLANES; plane++)
#pragma unroll
            for (int i = 0; i < std::decay_t<decltype(side)>::count; i++)
                side.issue(i, from + plane * s.plane, K - (int32_t)k0, buffer + plane * PLANE);
        if (++at.k == in_k) at.k = 0, at.segment++;
    };
    const auto copy_n = [&](int32_t s) { copies(cn, sn, next_n, s % BUFFERS * BUFFER); };
    const auto copy_m = [&](int32_t s) { copies(cm, sm, next_m, s % BUFFERS * BUFFER); };

    const auto piece_n = [&](int32_t s, int i, int k, int plane = 0) {
        return piece<NS, TN, STEP>(lds + s % BUFFERS * BUFFER + plane * PLANE, wn + i * 32, k);
    };
    const auto piece_m = [&](int32_t s, int j, int k, int plane = 0) {
        return piece<MS, TM, STEP>(lds + s % BUFFERS * BUFFER + plane * PLANE + TN * STEP * 2, wm + j * 32, k);
    };
    const auto meet = [] {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    const auto reads_there = [] { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };
    // and copies, but those of side N that were begun last
    const auto all_there = [](bool but_n) {
        if (but_n) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(decltype(cn)::count) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    };
    if constexpr (SM == 4) {
        static_assert(THREADS == 512);
        // Two wavefronts a SIMD, the second of each a phase behind: while one reads pieces, the other multiplies its own, and
        // they change over at a barrier.  A wavefront has two turns a step: it reads all its pieces of side N and half
        // of side M, then the other half.  So N is free for the step after the next when the second of the two has had its first
        // turn, and M with the step: the copies are begun half in each turn, three to six phases before the barrier at
        // which they are waited for.
        constexpr int H = SM / 2, KS = STEP / 16;
        const bool second = wave >= 4;
        if (steps > 0) {
            copy_n(0);
            copy_m(0);
            if (steps > 1) copy_n(1);
            all_there(steps > 1);
            meet();
        }
        if (second) meet();
        for (int32_t s = 0; s < steps; s++) {
            Bits8 pn[KS][SN], pm[KS][H];
#pragma unroll
            for (int turn = 0; turn < 2; turn++) {
#pragma unroll
                for (int k = 0; k < KS; k++) {
#pragma unroll
                    for (int i = 0; i < SN; i++)
                        if (turn == 0) pn[k][i] = piece_n(s, i, k * 16);
#pragma unroll
                    for (int j = 0; j < H; j++) pm[k][j] = piece_m(s, turn * H + j, k * 16);
                }
                if (turn == 0 && s + 1 < steps) copy_m(s + 1);
                if (turn == 1 && s + 2 < steps) copy_n(s);
                if (turn == 1 && second) all_there(s + 2 < steps);
                else reads_there();
                meet();
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int k = 0; k < KS; k++)
#pragma unroll
                    for (int i = 0; i < SN; i++)
#pragma unroll
                        for (int j = 0; j < H; j++) acc[i][turn * H + j] = multiply<T>(pn[k][i], pm[k][j], acc[i][turn * H + j]);
                __builtin_amdgcn_s_setprio(0);
                if (turn == 1 && !second) all_there(s + 2 < steps);
                meet();
            }
        }
        if (!second) meet();
    } else {
        // Two wavefronts a SIMD, and two workgroups a CU where there are as many.  The pieces of the next 16 k are read while these are
        // multiplied, the first of a step during the last of the step before: by then its copies are waited for, and with that
        // barrier every wavefront has read all of the buffer, which the next step to be copied goes to.
        Bits8 pn[2][PLANES][SN], pm[2][PLANES][SM];
        const auto read = [&](int to, int32_t s, int k) {
#pragma unroll
            for (int p = 0; p < PLANES; p++) {
#pragma unroll
                for (int i = 0; i < SN; i++) pn[to][p][i] = piece_n(s, i, k, p);
#pragma unroll
                for (int j = 0; j < SM; j++) pm[to][p][j] = piece_m(s, j, k, p);
            }
        };
        // fp32: the products of the parts but the first have sums of their own, in which they are not rounded to the first's last place
        Acc small[PLANES == 3 ? SN : 1][PLANES == 3 ? SM : 1];
        if constexpr (PLANES == 3)
#pragma unroll
            for (int i = 0; i < SN; i++)
#pragma unroll
                for (int j = 0; j < SM; j++)
#pragma unroll
                    for (int e = 0; e < 16; e++) small[i][j][e] = 0.0f;
        const auto products = [&](int of) {
#pragma unroll
            for (int q = PLANES == 3 ? 0 : 5; q < 6; q++) {       // parts (2,0) (0,2) (1,1) (1,0) (0,1) (0,0)
                const int n = (0x001102 >> (4 * q)) & 15, m = (0x010120 >> (4 * q)) & 15;
#pragma unroll
                for (int i = 0; i < SN; i++)
#pragma unroll
                    for (int j = 0; j < SM; j++) {
                        Acc &c = q < 5 ? small[PLANES == 3 ? i : 0][PLANES == 3 ? j : 0] : acc[i][j];
                        c = multiply<T>(pn[of][n][i], pm[of][m][j], c);
                    }
            }
        };
        const auto copy = [&](int32_t s) {
            copy_n(s);
            copy_m(s);
        };
        static constexpr int kCopies = PLANES * (decltype(cn)::count + decltype(cm)::count);       // a wavefront's in each step
        const auto there = [](int32_t later) {               // reads, and copies but those of the `later` last steps
            if (BUFFERS > 2 && later >= 3) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(3 * kCopies) : "memory");
            else if (BUFFERS > 2 && later == 2) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * kCopies) : "memory");
            else if (later == 1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kCopies) : "memory");
            else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        };
        if (steps > 0) {
            for (int32_t s = 0; s < min(steps, BUFFERS); s++) copy(s);
            there(min(steps, BUFFERS) - 1);
            meet();
            read(0, 0, 0);
        }
        for (int32_t s = 0; s < steps; s++) {
#pragma unroll
            for (int k = 0; k < STEP / 16; k++) {
                if (k + 1 < STEP / 16) {
                    read((k + 1) % 2, s, (k + 1) * 16);
                } else {
                    // also after the last step, and what is read then is not used: behind a branch around the reads the compiler
                    // would wait for all that are on their way
                    there(min(steps - 2 - s, BUFFERS - 2));
                    meet();
                    if (s + BUFFERS < steps) copy(s);
                    read(0, s + 1, 0);
                }
                __builtin_amdgcn_sched_barrier(0);       // left to itself the compiler puts the reads after the products
                products(k % 2);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if constexpr (PLANES == 3)
#pragma unroll
            for (int i = 0; i < SN; i++)
#pragma unroll
                for (int j = 0; j < SM; j++) acc[i][j] += small[i][j];
    }

    // The result goes through LDS, a wavefront's rows of 64 n at a time, each by itself: an accumulator's lanes have four n of 32 rows,
    // a store of which would be 32 pieces of as many lines; after it eight lanes have a row's 64.
    static_assert(SN == 2);
    using Result = std::conditional_t<WHAT == Product::parts, ElemF32, T>;
    using E = typename Result::elem;
    constexpr bool NARROW = sizeof(E) == 2 && WHAT != Product::gated && WHAT != Product::gated_gradient;      // staged as stored
#pragma unroll
    for (int j = 0; j < SM; j++) {
        CCDC_LDS unsigned char *stage = lds + (SM > 1 ? wave * 2 + j % 2 : wave) * (NARROW ? 4096 : 8192);
        static_assert(BUFFERS * BUFFER >= WN * WM * (SM > 1 ? 2 : 1) * (NARROW ? 4096 : 8192));
#pragma unroll
        for (int i = 0; i < SN; i++)
#pragma unroll
            for (int g = 0; g < 4; g++) {
                const uint32_t row = lane % 32, four = i * 8 + g * 2 + lane / 32;
                if constexpr (NARROW) {
                    typedef E Four __attribute__((ext_vector_type(4)));
                    Four v;
#pragma unroll
                    for (int e = 0; e < 4; e++) v[e] = narrow<T>(acc[i][j][4 * g + e]);
                    *(CCDC_LDS Four *)(stage + row * 128 + (four / 2 ^ row / 2 % 8) * 16 + four % 2 * 8) = v;
                } else {
                    typedef float Four __attribute__((ext_vector_type(4)));
                    Four v;
#pragma unroll
                    for (int e = 0; e < 4; e++) v[e] = acc[i][j][4 * g + e];
                    *(CCDC_LDS Four *)(stage + row * 256 + (four ^ row % 16) * 16) = v;
                }
            }
        // numbers 8 pack ... 8 pack + 7 of a row
        const auto staged = [&](uint32_t row, uint32_t pack) {
            typedef float Four __attribute__((ext_vector_type(4)));
            Eight v;
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const Four f = *(CCDC_LDS Four *)(stage + row * 256 + ((pack * 2 + h) ^ row % 16) * 16);
#pragma unroll
                for (int e = 0; e < 4; e++) v.v[4 * h + e] = f[e];
            }
            return v;
        };
        constexpr int LANES = GATED ? 4 : 8;              // that have a row: 32 of a and of u, or 64
#pragma unroll
        for (int q = 0; q < 32 * LANES / 64; q++) {
            CCDC_AS_WRITTEN
            const uint32_t row = q * (64 / LANES) + lane / LANES, pack = lane % LANES;
            const int32_t m = tile_m + wm + j * 32 + row;
            if (m >= a.rows_m) continue;
            if constexpr (GATED) {
                const int32_t f = tile_n + wn / 2 + pack * 8;
                if (f >= a.ldh) continue;
                const Eight va = staged(row, pack), vu = staged(row, 4 + pack);
                Eight h, P, Q, keep;
                if (a.drop.threshold) {
                    const RowOf of = a.row_of[m];
                    keep = dropout_factors(a.drop, of.id, of.token, f / 8);
                }
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    float value, slope;
                    activate<T>(a.activation, va.v[e], value, slope);
                    h.v[e] = value * vu.v[e], P.v[e] = slope * vu.v[e], Q.v[e] = value;
                    P.v[e] += 0.0f;           // (no negative zero: that is what is taken out)
                    if (a.drop.threshold) {
                        h.v[e] = kept(h.v[e], keep.v[e]), Q.v[e] = kept(Q.v[e], keep.v[e]);
                        P.v[e] = keep.v[e] != 0.0f ? P.v[e] * keep.v[e] : kTakenOut;
                    }
                    if (f + e >= a.rows_n) h.v[e] = P.v[e] = Q.v[e] = 0.0f;
                }
                const int64_t at = (int64_t)m * a.ldh + f;
                // 16-bit modes: rounded to the mode's format, as the gradients of a and u are, since that is what the matrix
                // instructions multiply (in parts, as fp32 has it, three or six times the products).  Results are 1.4 times as far
                // off as by their own rounding alone; binary16 has an infinity above 65504.
                store_side<T>(a.h + at, a.plane_h, h);
                if (a.P) {
                    store_eight<ElemF32>(a.P + at, P, 8);
                    store_eight<ElemF32>(a.Q + at, Q, 8);
                }
            } else {
                const int32_t n = tile_n + wn + pack * 8;
                if constexpr (WHAT == Product::gated_gradient) {
                    if (n >= a.ldh) continue;
                    const Eight v = staged(row, pack);
                    const int64_t at = (int64_t)m * a.ldh + n;
                    const Eight P = load_eight<ElemF32>(a.P + at, 8), Q = load_eight<ElemF32>(a.Q + at, 8);
                    Eight da, du;
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        // nothing comes of a value that was taken out, whatever its gradient (an infinity or no number too)
                        const bool none = n + e >= a.rows_n || __float_as_uint(P.v[e]) == __float_as_uint(kTakenOut);
                        da.v[e] = none ? 0.0f : v.v[e] * P.v[e], du.v[e] = none ? 0.0f : v.v[e] * Q.v[e];
                    }
                    uint16_t *to = a.h + (int64_t)m * 2 * a.ldh + n;
                    store_side<T>(to, a.plane_h, da);
                    store_side<T>(to + a.second_h, a.plane_h, du);
                } else {
                    if (n >= a.rows_n) continue;
                    E *to = (E *)a.c + file * a.file_c + half * a.half_c + (int64_t)m * a.ldc + n;
                    if constexpr (NARROW) {
                        const Bits8 v = *(CCDC_LDS Bits8 *)(stage + row * 128 + (pack ^ row / 2 % 8) * 16);
                        const int valid = fresh(a.rows_n - n);
                        if (valid >= 8) {
                            store_any<Bits8, E>(to, v);
                        } else {
#pragma unroll
                            for (int e = 0; e < 8; e++)
                                if (e < valid) to[e] = (E)v[e];
                        }
                    } else {
                        store_eight<Result>(to, staged(row, pack), a.rows_n - n);
                    }
                }
            }
        }
    }
}

template <class T, Product WHAT, int WN, int WM, int SN, int SM, int BUFFERS>
int launch(ProductArgs a, hipStream_t st)
{
    a.tiles_n = cdiv(a.rows_n, WN * SN * 32 / (WHAT == Product::gated ? 2 : 1));
    a.tiles_m = cdiv(a.rows_m, WM * SM * 32);
    const uint64_t tiles = (uint64_t)a.tiles_n * a.tiles_m * a.files * a.halves;
    if (!fits_launch(tiles * 64 * WN * WM)) return CCDC_ESIZE;
    k_product<T, WHAT, WN, WM, SN, SM, BUFFERS><<<(uint32_t)tiles, 64 * WN * WM, 0, st>>>(a);
    return launched();
}

// Tiles of 256 x 256, one a CU, or of 128 x 128, two (16-bit numbers), by the rounds of them that the chip's 256 CUs make.  A round of large
// ones is twice the work of a round of small ones in 1.75 of the time (2048 x 4160 bf16, a and u: 462 large tiles 178 us, 910 small ones
// 102).  A tile of a gradient of weights is short, as its file is, and what comes before and after the products counts: with
// 28 files of 64 tokens the small tiles took 0.90 of the time, of 128 1.03, of 512 1.25; 515 x 1333, where the large ones are a
// quarter past the edge, 64 tokens 0.69, 256 0.86.
template <Product WHAT>
bool large_tiles(const ProductArgs &a)
{
    const auto rounds = [&](uint32_t size, uint32_t at_once) {
        return (double)cdiv((uint64_t)cdiv(a.rows_n, WHAT == Product::gated ? size / 2 : size) * cdiv(a.rows_m, size) * a.files * a.halves, at_once);
    };
    double time = 1.75;
    if (WHAT == Product::weight_gradient) time = a.K < 128 ? 2.2 : a.K < 256 ? 1.9 : 1.6;
    return rounds(256, 256) * time <= rounds(128, 512);
}

template <class T, Product WHAT>
int by_tile(const ProductArgs &a, hipStream_t st)
{
    if constexpr (T::planes == 3) {
        // fp32: 128 x 256 or 128 x 128, one a CU; a round of the former has twice the work in 1.45 to 1.7 of the time (4040 tokens,
        // 1024 x 2600: a and u in 3 rounds 285 us, 6 of small ones 336; dx, whose large tiles are half a round, 416 and 282).  It does not look at the files' tokens:
        // where they are few a tile has one step, and a training step takes longer than one of the library's fp32 products (20 files of 8
        // tokens 663 us and 425, 64 of 8 1060 and 858; 20 of 64 815 and 932).
        const auto rounds = [&](uint32_t m) {
            return (double)cdiv((uint64_t)cdiv(a.rows_n, WHAT == Product::gated ? 64 : 128) * cdiv(a.rows_m, m) * a.files * a.halves, 256);
        };
        if (WHAT != Product::parts && rounds(256) * 1.6 <= rounds(128)) return launch<T, WHAT, 2, 4, 2, 2, 2>(a, st);
        return launch<T, WHAT, 2, 4, 2, 1, 3>(a, st);
    } else if constexpr (WHAT == Product::parts) {
        return launch<T, WHAT, 2, 4, 2, 1, 4>(a, st);
    } else {
        if (large_tiles<WHAT>(a)) return launch<T, WHAT, 4, 2, 2, 4, 2>(a, st);
        const uint64_t small = (uint64_t)cdiv(a.rows_n, WHAT == Product::gated ? 64 : 128) * cdiv(a.rows_m, 128) * a.files * a.halves;
        if (small > 256) return launch<T, WHAT, 2, 4, 2, 1, 2>(a, st);
        return launch<T, WHAT, 2, 4, 2, 1, 4>(a, st);         // one a CU: with its LDS, more of a tile on its way
    }
}

template <class T>
int by_product(Product what, const ProductArgs &a, hipStream_t st)
{
    switch (what) {
    case Product::gated: return by_tile<T, Product::gated>(a, st);
    case Product::plain: return by_tile<T, Product::plain>(a, st);
    case Product::parts: return by_tile<T, Product::parts>(a, st);
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
