// Products of matrices in 8 bits, for more than a few rows.
//
// A workgroup makes a tile of C, its wavefronts 32 x 32 pieces of it by v_mfma_scale_f32_32x32x64, rows of N as the instruction's
// rows.  A step is one block of 128 of both sides, so each row has one scale in it, and 128 bytes.  Steps are copied into LDS past the
// registers while those before are computed on; the scales of four steps are a word a row and are copied with the first of them.
// Bytes lie in LDS as [row][128], a row's packs of 16 in an order of its own (product.hip: what a wavefront reads together is in
// different banks).  A lane has 32 of a row's 64 k of an instruction, the same ones on both sides, which is all that a
// product asks for.
#include <algorithm>

#include "eight.hpp"

namespace {
using namespace ccdc;

typedef float Acc __attribute__((ext_vector_type(16)));
#define CCDC_LDS __attribute__((address_space(3)))

// Copies 16 (4) bytes a lane to LDS, lane after lane from byte `to` on.  The compiler does not count these: every step's are
// waited for in one place.
__device__ __forceinline__ void copy_to_lds(uint32_t to, const void *base, uint32_t offset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :: "s"(to), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ void copy_words_to_lds(uint32_t to, const void *base, uint32_t offset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
                 :: "s"(to), "v"(offset), "s"(base) : "memory");
}

// Place in its row of pack `pack` (16 bytes, eight a row).
__device__ __forceinline__ uint32_t pack_place(uint32_t row, uint32_t pack) { return pack ^ (row / 2 % 8); }

// The copies of one side that a wavefront makes in each step.
template <int ROWS, int THREADS>
struct Copies {
    static constexpr int count = ROWS * 8 / THREADS;
    const uint8_t *base[count];           // the same for all lanes
    uint32_t offset[count];               // bytes, a lane's own
    uint32_t to;                          // byte in LDS of the first

    __device__ __forceinline__ void set(const uint8_t *side, int32_t ld, int32_t row0, int32_t rows, uint32_t lds)
    {
        const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
        to = lds + wave * 1024;
#pragma unroll
        for (int i = 0; i < count; i++) {
            const int32_t r = (i * THREADS + wave * 64) / 8, from = min(row0 + r, rows - 1);
            const int32_t at = min(from + (int32_t)(lane / 8), rows - 1) - from;
            base[i] = side + (int64_t)from * ld;
            offset[i] = (uint32_t)(at * ld) + pack_place(r + lane / 8, lane % 8) * 16;
        }
    }
    __device__ __forceinline__ void issue(int32_t step, uint32_t buffer) const
    {
#pragma unroll
        for (int i = 0; i < count; i++)
            copy_to_lds(__builtin_amdgcn_readfirstlane(to + buffer + i * THREADS * 16), base[i] + (int64_t)step * 128, offset[i]);
    }
};

// The numbers of 64 k (half 0 or 1 of a step) of 32 rows from row0 on, as a lane has them.
__device__ __forceinline__ Bytes32 piece(CCDC_LDS unsigned char *lds, int row0, int half)
{
    const uint32_t lane = threadIdx.x % 64, row = row0 + lane % 32, pack = half * 4 + lane / 32;
    CCDC_LDS unsigned char *p = lds + row * 128;
    return both(*(CCDC_LDS Bytes16 *)(p + pack_place(row, pack) * 16), *(CCDC_LDS Bytes16 *)(p + pack_place(row, pack + 2) * 16));
}

// SN x SM pieces of 32 x 32 over 64 k.
template <class T, int SN, int SM, int FROM, int COUNT>
__device__ __forceinline__ void multiply(Acc (&acc)[SN][SM], const Bytes32 (&n)[SN], const Bytes32 (&m)[COUNT], const int (&sn)[SN], const int (&sm)[SM])
{
    if constexpr (T::planes == 1) {
#pragma unroll
        for (int i = 0; i < SN; i++)
#pragma unroll
            for (int j = 0; j < COUNT; j++)
                acc[i][FROM + j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(n[i], m[j], acc[i][FROM + j], 0, 0, 0, sn[i], 0, sm[FROM + j]);
    } else {
        // fp32 results: as bfloat16 with the scales (eight.hpp)
#pragma unroll
        for (int q = 0; q < 4; q++) {
            Wide8 wn[SN], wm[COUNT];
#pragma unroll
            for (int i = 0; i < SN; i++) wn[i] = wide(n[i][2 * q], n[i][2 * q + 1], power(sn[i]));
#pragma unroll
            for (int j = 0; j < COUNT; j++) wm[j] = wide(m[j][2 * q], m[j][2 * q + 1], power(sm[FROM + j]));
#pragma unroll
            for (int i = 0; i < SN; i++)
#pragma unroll
                for (int j = 0; j < COUNT; j++) acc[i][FROM + j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wn[i], wm[j], acc[i][FROM + j], 0, 0, 0);
        }
    }
}

// 32 x 32 sums from memory, a lane's row of either side given, as `multiply` adds them, where scales leave bfloat16's range.
__device__ __forceinline__ Acc sum_in_turns(const Product8Args &a, int32_t row_n, int32_t row_m)
{
    const uint32_t pack = threadIdx.x % 64 / 32 * 16;
    const uint8_t *n = a.n + (int64_t)row_n * a.ld + pack, *m = a.m + (int64_t)row_m * a.ld + pack;
    const uint8_t *n_scale = a.n_scale + (int64_t)row_n * a.ld_scale, *m_scale = a.m_scale + (int64_t)row_m * a.ld_scale;
    Acc sum = {};
#pragma unroll 1
    for (int32_t s = 0; s < a.blocks * 2; s++) {              // halves of a block, as `piece` has them
        const Bytes32 bn = both(*(const Bytes16 *)(n + (int64_t)s * 64), *(const Bytes16 *)(n + (int64_t)s * 64 + 32));
        const Bytes32 bm = both(*(const Bytes16 *)(m + (int64_t)s * 64), *(const Bytes16 *)(m + (int64_t)s * 64 + 32));
#pragma unroll 1
        for (int turn = 0; turn < kScaleTurns; turn++) {
            const ScaleInTurn sn = scale_in_turn(n_scale[s / 2], true, turn), sm = scale_in_turn(m_scale[s / 2], false, turn);
#pragma unroll
            for (int q = 0; q < 4; q++)
                sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wide_in_turn(bn[2 * q], bn[2 * q + 1], sn), wide_in_turn(bm[2 * q], bm[2 * q + 1], sm), sum, 0, 0, 0);
        }
    }
    return sum;
}

// WN x WM wavefronts, each SN x SM pieces; BUFFERS steps in LDS.
template <class T, int WN, int WM, int SN, int SM, int BUFFERS>
__global__ __launch_bounds__(64 * WN * WM) void k_product8(const Product8Args a)
{
    constexpr int THREADS = 64 * WN * WM, TN = WN * SN * 32, TM = WM * SM * 32, BUFFER = (TN + TM) * 128, SCALES = (TN + TM) * 4;
    __shared__ __attribute__((aligned(1024))) unsigned char memory[BUFFERS * BUFFER + 2 * SCALES];
    CCDC_LDS unsigned char *lds = (CCDC_LDS unsigned char *)memory;
    const uint32_t lds_at = (uint32_t)(uintptr_t)lds;

    // Tiles as in product.hip: an XCD takes a contiguous range of them, in groups of eight rows of tiles.
    constexpr uint32_t kGroup = 8;
    const uint32_t t = xcd_contiguous(blockIdx.x, gridDim.x), in_group = kGroup * a.tiles_n;
    const uint32_t group = t / in_group, rows_in = min(a.tiles_m - group * kGroup, kGroup), in = t - group * in_group;
    const int32_t tile_m = (group * kGroup + in % rows_in) * TM, tile_n = in / rows_in * TN;

    Copies<TN, THREADS> cn;
    Copies<TM, THREADS> cm;
    cn.set(a.n, a.ld, tile_n, a.rows_n, lds_at);
    cm.set(a.m, a.ld, tile_m, a.rows_m, lds_at + TN * 128);
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int wn = wave % WN * SN * 32, wm = wave / WN * SM * 32;

    // The words of 64 rows that a wavefront copies every four steps; with fewer words than wavefronts have lanes some are copied twice.
    const uint32_t word = wave * 64 % (TN + TM);
    const bool of_n = word < (uint32_t)TN;
    const int32_t word_rows = of_n ? a.rows_n : a.rows_m, word_from = min(of_n ? tile_n + (int32_t)word : tile_m + (int32_t)word - TN, word_rows - 1);
    const uint8_t *word_base = (of_n ? a.n_scale : a.m_scale) + (int64_t)word_from * a.ld_scale;
    const uint32_t word_offset = (uint32_t)((min(word_from + lane, word_rows - 1) - word_from) * a.ld_scale);
    static_assert((TN + TM) % 64 == 0 && TN + TM <= THREADS && TN % 64 == 0);

    Acc acc[SN][SM];
#pragma unroll
    for (int i = 0; i < SN; i++)
#pragma unroll
        for (int j = 0; j < SM; j++)
#pragma unroll
            for (int e = 0; e < 16; e++) acc[i][j][e] = 0.0f;

    const int32_t steps = a.blocks;
    // side N's come first, with the words where a step is the first of four: what is waited for below counts the copies of a side
    // or of a step, and these are one more, so that a little more is waited for
    const auto copy_n = [&](int32_t s) {
        if (s % 4 == 0)
            copy_words_to_lds(__builtin_amdgcn_readfirstlane(lds_at + BUFFERS * BUFFER + s / 4 % 2 * SCALES + word * 4), word_base + s, word_offset);
        cn.issue(s, s % BUFFERS * BUFFER);
    };
    const auto copy_m = [&](int32_t s) { cm.issue(s, s % BUFFERS * BUFFER); };
    const auto piece_n = [&](int32_t s, int i, int half) { return piece(lds + s % BUFFERS * BUFFER, wn + i * 32, half); };
    const auto piece_m = [&](int32_t s, int j, int half) { return piece(lds + s % BUFFERS * BUFFER + TN * 128, wm + j * 32, half); };
    const auto scale_at = [&](int32_t s, int row) {
        return (int)*(lds + BUFFERS * BUFFER + s / 4 % 2 * SCALES + (row + lane % 32) * 4 + s % 4);
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
    int sn[SN], sm[SM];
    ScalesSeen seen;
    if constexpr (SM == 4) {
        static_assert(THREADS == 512);
        // Two wavefronts a SIMD, the second of each a phase behind, in turns at reading pieces and multiplying them (product.hip).
        constexpr int H = SM / 2;
        const bool second = wave >= 4;
        copy_n(0);
        copy_m(0);
        if (steps > 1) copy_n(1);
        all_there(steps > 1);
        meet();
        if (second) meet();
        for (int32_t s = 0; s < steps; s++) {
            Bytes32 pn[2][SN], pm[2][H];
#pragma unroll
            for (int turn = 0; turn < 2; turn++) {
                if (turn == 0) {
#pragma unroll
                    for (int i = 0; i < SN; i++) sn[i] = scale_at(s, wn + i * 32);
#pragma unroll
                    for (int j = 0; j < SM; j++) sm[j] = scale_at(s, TN + wm + j * 32);
                }
#pragma unroll
                for (int k = 0; k < 2; k++) {
#pragma unroll
                    for (int i = 0; i < SN; i++)
                        if (turn == 0) pn[k][i] = piece_n(s, i, k);
#pragma unroll
                    for (int j = 0; j < H; j++) pm[k][j] = piece_m(s, turn * H + j, k);
                }
                if (turn == 0 && s + 1 < steps) copy_m(s + 1);
                if (turn == 1 && s + 2 < steps) copy_n(s + 2);
                if (turn == 1 && second) all_there(s + 2 < steps);
                else reads_there();
                meet();
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int k = 0; k < 2; k++) {
                    if (turn == 0) multiply<T, SN, SM, 0, H>(acc, pn[k], pm[k], sn, sm);
                    else multiply<T, SN, SM, H, H>(acc, pn[k], pm[k], sn, sm);
                }
                __builtin_amdgcn_s_setprio(0);
                if (turn == 1 && !second) all_there(s + 2 < steps);
                meet();
            }
        }
        if (!second) meet();
    } else {
        // Two wavefronts a SIMD, and two workgroups a CU where there are as many: the pieces of the next 64 k are read while
        // these are multiplied (product.hip).
        Bytes32 pn[2][SN], pm[2][SM];
        int next_n[SN], next_m[SM];
        const auto read = [&](int to, int32_t s, int half) {
#pragma unroll
            for (int i = 0; i < SN; i++) pn[to][i] = piece_n(s, i, half);
#pragma unroll
            for (int j = 0; j < SM; j++) pm[to][j] = piece_m(s, j, half);
            if (half == 0) {
#pragma unroll
                for (int i = 0; i < SN; i++) next_n[i] = scale_at(s, wn + i * 32);
#pragma unroll
                for (int j = 0; j < SM; j++) next_m[j] = scale_at(s, TN + wm + j * 32);
            }
        };
        const auto copy = [&](int32_t s) {
            copy_n(s);
            copy_m(s);
        };
        static constexpr int kCopies = decltype(cn)::count + decltype(cm)::count;       // a wavefront's in each step
        const auto there = [](int32_t later) {               // reads, and copies but those of the `later` last steps
            if (BUFFERS > 2 && later >= 3) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(3 * kCopies) : "memory");
            else if (BUFFERS > 2 && later == 2) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * kCopies) : "memory");
            else if (later == 1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kCopies) : "memory");
            else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        };
        for (int32_t s = 0; s < min(steps, BUFFERS); s++) copy(s);
        there(min(steps, BUFFERS) - 1);
        meet();
        read(0, 0, 0);
        for (int32_t s = 0; s < steps; s++) {
#pragma unroll
            for (int i = 0; i < SN; i++) sn[i] = next_n[i];
#pragma unroll
            for (int j = 0; j < SM; j++) sm[j] = next_m[j];
            read(1, s, 1);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (T::planes == 3) {
#pragma unroll
                for (int i = 0; i < SN; i++) seen.see(sn[i]);
#pragma unroll
                for (int j = 0; j < SM; j++) seen.see(sm[j]);
            }
            multiply<T, SN, SM, 0, SM>(acc, pn[0], pm[0], sn, sm);
            __builtin_amdgcn_sched_barrier(0);
            // also after the last step, and what is read then is not used (product.hip)
            there(min(steps - 2 - s, BUFFERS - 2));
            meet();
            if (s + BUFFERS < steps) copy(s + BUFFERS);
            read(0, s + 1, 0);
            __builtin_amdgcn_sched_barrier(0);
            multiply<T, SN, SM, 0, SM>(acc, pn[1], pm[1], sn, sm);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // what was read last is not used, and other wavefronts' reads of it are over before it is written over
    reads_there();
    meet();
    if constexpr (T::planes == 3)
        if (seen.others())
#pragma unroll
            for (int i = 0; i < SN; i++)
#pragma unroll
                for (int j = 0; j < SM; j++)
                    acc[i][j] = sum_in_turns(a, min(tile_n + wn + i * 32 + lane % 32, a.rows_n - 1), min(tile_m + wm + j * 32 + lane % 32, a.rows_m - 1));

    // The result goes through LDS, a wavefront's rows of 64 n at a time, each by itself (product.hip).
    static_assert(SN == 2);
    using E = typename T::elem;
    constexpr bool NARROW = sizeof(E) == 2;
#pragma unroll
    for (int j = 0; j < SM; j++) {
        CCDC_LDS unsigned char *stage = lds + (SM > 1 ? wave * 2 + j % 2 : wave) * (NARROW ? 4096 : 8192);
        static_assert(BUFFERS * BUFFER >= WN * WM * (SM > 1 ? 2 : 1) * (NARROW ? 4096 : 8192));
        typedef E Four __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int i = 0; i < SN; i++)
#pragma unroll
            for (int g = 0; g < 4; g++) {
                const uint32_t row = lane % 32, four = i * 8 + g * 2 + lane / 32;
                Four v;
#pragma unroll
                for (int e = 0; e < 4; e++) v[e] = narrow<T>(acc[i][j][4 * g + e]);
                if constexpr (NARROW) *(CCDC_LDS Four *)(stage + row * 128 + (four / 2 ^ row / 2 % 8) * 16 + four % 2 * 8) = v;
                else *(CCDC_LDS Four *)(stage + row * 256 + (four ^ row % 16) * 16) = v;
            }
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const uint32_t row = q * 8 + lane / 8, pack = lane % 8;
            const int32_t m = tile_m + wm + j * 32 + row, n = tile_n + wn + pack * 8;
            if (m >= a.rows_m || n >= a.rows_n) continue;
            E *to = (E *)a.c + (int64_t)m * a.ldc + n;
            if constexpr (NARROW) {
                typedef E Packed __attribute__((ext_vector_type(8)));
                const Packed v = *(CCDC_LDS Packed *)(stage + row * 128 + (pack ^ row / 2 % 8) * 16);
                const int valid = fresh(a.rows_n - n);
                if (valid >= 8) {
                    store_any<Packed, E>(to, v);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; e++)
                        if (e < valid) to[e] = v[e];
                }
            } else {
                Eight v;
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const Four f = *(CCDC_LDS Four *)(stage + row * 256 + ((pack * 2 + h) ^ row % 16) * 16);
#pragma unroll
                    for (int e = 0; e < 4; e++) v.v[4 * h + e] = f[e];
                }
                store_eight<T>(to, v, a.rows_n - n);
            }
        }
    }
}

template <class T, int WN, int WM, int SN, int SM, int BUFFERS>
int launch(Product8Args a, hipStream_t st)
{
    const uint64_t tiles_n = cdiv(a.rows_n, WN * SN * 32), tiles_m = cdiv(a.rows_m, WM * SM * 32);
    if (!fits_launch(tiles_n * tiles_m * 64 * WN * WM)) return CCDC_ESIZE;
    a.tiles_n = (int32_t)tiles_n, a.tiles_m = (int32_t)tiles_m;
    k_product8<T, WN, WM, SN, SM, BUFFERS><<<(uint32_t)(tiles_n * tiles_m), 64 * WN * WM, 0, st>>>(a);
    return launched();
}

// The tile by the rounds of them that the chip's 256 CUs make, at what a step of a round took (us; 65 to 8192 rows of 2048 and 4096 columns,
// 4096 to 11264 outputs, bf16): 256 x 256, one a CU, 1.65; 128 x 128 two a CU 1.2, or one with twice the steps in LDS 0.72; 64 outputs x 128
// rows, one a CU, 0.59; 64 x 64, two a CU, 0.66, of one 0.5.  333 rows of 2048 x 4160: 9.1 us by 64 x 128, by 128 x 128 11.5; 64 rows of 4096
// x 11264 16.0 by 64 x 64, 21.4; 1024 rows 56 by the largest, 68 and 74 by 128 x 128.
// fp32 results, of half the rate, go by the same costs without the largest: of 14 shapes from 65 to 8192 rows no tile was more than 3 % faster than
// the one taken (333 rows 14.1 us by 64 x 128, by 128 x 128 18.5; 8192 x 4096 x 11264 680 by two 128 x 128 a CU, 807 by one, 957 by 64 x 64), but for
// 1024 x 4096 x 11264, 112 by one 128 x 128 a CU and 96 by two.
template <class T>
int run_product8(const Product8Args &a, hipStream_t st)
{
    const auto tiles = [&](uint32_t n, uint32_t m) { return (uint64_t)cdiv(a.rows_n, n) * cdiv(a.rows_m, m); };
    const double largest = cdiv(tiles(256, 256), 256) * 1.65, two = cdiv(tiles(128, 128), 512) * 1.2, one = cdiv(tiles(128, 128), 256) * 0.72;
    const double tall = cdiv(tiles(64, 128), 256) * 0.59, small = tiles(64, 64) <= 256 ? 0.5 : cdiv(tiles(64, 64), 512) * 0.66;
    const double least = std::min(std::min(small, tall), std::min(one, two));
    if constexpr (T::planes == 1)                     // (in fp32 a large tile's pieces as bfloat16 are more registers than there are)
        if (largest <= least) return launch<T, 4, 2, 2, 4, 2>(a, st);
    if (small == least) return launch<T, 1, 2, 2, 1, 4>(a, st);
    if (tall == least) return launch<T, 1, 4, 2, 1, 4>(a, st);
    if (one == least) return launch<T, 2, 4, 2, 1, 4>(a, st);
    return launch<T, 2, 4, 2, 1, 2>(a, st);
}

}  // namespace

namespace ccdc {

int tiled_product8(const ccdc_block_t *b, const Product8Args &a, hipStream_t st) { CCDC_BY_ELEM(b, (run_product8<T>(a, st))); }

}  // namespace ccdc
