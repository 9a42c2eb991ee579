// The largest logits of rows, in order, and the logarithm of what all others come to.
//
// A workgroup has a row, held in registers where it fits.  The k-th largest of the threads' own largest values is a bound that at
// least k values reach and few more: with each thread's value in LDS, sixteen bounds at a time are counted by ballots, so five rounds find
// twenty bits of it.  What reaches it is put into a list in LDS, whatever the order, and ranked there: as keys of 64 bits, value then
// column, no two are equal, so the order is one.  Where the list is long for its k (short rows of which much is wanted) the k-th
// largest in it is found first, by ballots, bit by bit.  Where there is no room for all that reaches the bound (many equal values, those
// of a mask by the lowest number among them; rows of 513 to 1024 columns with k above the 64 threads that they have, which give no
// bound then) the row is counted again by digits of eight bits of those keys, values first and then columns, until what is left has room.
#include "vocabulary.hpp"

namespace {
using namespace ccdc;

struct TopArgs {
    const void *z;
    int32_t *index;
    float *value, *rest;
    int64_t ldz;
    int32_t columns, k;
    float per_T;
};

constexpr float kLog2e = 1.44269504f;

// A number that grows with v, and 0 for what is never listed: -infinity and NaNs.
__device__ __forceinline__ uint32_t ordered(float v)
{
    const uint32_t u = __float_as_uint(v + 0.0f);             // (no negative zero)
    return v > -INFINITY ? u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u) : 0u;
}
__device__ __forceinline__ float value_of(uint32_t key)
{
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

constexpr int kFew = 96;                          // of the list: not worth a search of the k-th

template <class T, int WAVES, int PACKS>
__global__ __launch_bounds__(64 * WAVES) void k_top(const TopArgs a)
{
    constexpr int THREADS = 64 * WAVES, DIGITS = 16 / WAVES, ROUNDS = std::is_same<T, ElemBF16>::value ? 4 : 5;
    constexpr int kRoom = WAVES == 1 ? 512 : WAVES <= 4 ? 1024 : 2048;  // of the list
    __shared__ double part[2 * WAVES];
    __shared__ uint32_t largest[THREADS];
    __shared__ int32_t counts[2][16];
    __shared__ __attribute__((aligned(16))) uint64_t found[kRoom + 8];
    __shared__ int32_t used;
    __shared__ uint64_t last;
    OverRow<WAVES> over{part};
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const auto none = [](int32_t) { return 0u; };
    if (WAVES > 1 || PACKS > 1) __builtin_assume(a.columns >= 8);     // (by_columns; shorter rows' loads are many registers)
    Row<T, WAVES, PACKS> z;
    z.load(a.z, row * a.ldz, a.columns);
    float most = -INFINITY, pack_most[PACKS ? PACKS : 1] = {};
    const auto most_of = [&](const Eight &v) {
        float pack = v.v[0];
#pragma unroll
        for (int i = 1; i < 8; i++) pack = fmaxf(pack, v.v[i]);
        most = fmaxf(most, pack);
        return pack;
    };
    if constexpr (PACKS > 0) {
        int i = 0;
        z.template hide_held<true>(none, [&](const Eight &v) { pack_most[i++] = most_of(v); });
    } else {
        z.each(none, [&](const Eight &v, int32_t, uint32_t) { most_of(v); });
    }
    const uint32_t own = ordered(most);
    uint32_t bound = 0;
    if constexpr (WAVES == 1) {
#pragma unroll
        for (int bit = 31; bit > 31 - 4 * ROUNDS; bit--) {
            const uint32_t next = bound | 1u << bit;
            if ((int)__popcll(__ballot(own >= next)) >= a.k) bound = next;
        }
        if (threadIdx.x == 0) used = 0, last = 0;
        __syncthreads();
    } else {
        largest[threadIdx.x] = own;
        if (threadIdx.x == 0) used = 0, last = 0;
        __syncthreads();
        uint32_t all[WAVES];
#pragma unroll
        for (int i = 0; i < WAVES; i++) all[i] = largest[i * 64 + lane];
#pragma unroll
        for (int round = 0; round < ROUNDS; round++) {
            const int shift = 28 - 4 * round;
#pragma unroll
            for (int d = 0; d < DIGITS; d++) {
                const int digit = wave * DIGITS + d;
                const uint32_t from = bound | (uint32_t)digit << shift;
                int count = 0;
#pragma unroll
                for (int i = 0; i < WAVES; i++) count += __popcll(__ballot(all[i] >= from));
                if (lane == 0) counts[round % 2][digit] = count;
            }
            __syncthreads();
            const uint32_t reach = (uint32_t)__ballot(lane < 16 && counts[round % 2][lane % 16] >= a.k) | 1u;
            bound |= (uint32_t)(31 - __builtin_clz(reach)) << shift;
        }
    }
    // the same as a number: at least the lowest, so that -infinity and NaNs stay out
    const float least_wanted = bound > 0x00800000u ? value_of(bound) : kLowest;

    const auto put = [&](float v, int32_t c) {
        const int to = atomicAdd(&used, 1);
        if (to < kRoom) found[to] = (uint64_t)ordered(v) << 32 | (0xFFFFFFFFu - (uint32_t)c);
    };
    if (most >= least_wanted) {
        int i = 0;
        z.each(none, [&](const Eight &v, int32_t c, uint32_t) {
            bool any = true;
            if constexpr (PACKS > 0) any = pack_most[i++] >= least_wanted;
            if (any)
#pragma unroll
                for (int e = 0; e < 8; e++)
                    if (v.v[e] >= least_wanted) put(v.v[e], c + e);
        });
    }
    __syncthreads();
    int32_t n = used;
    if (n > kRoom) {                              // (the same for all threads)
        // as numbers of 56 bits; the k-th's from the highest digit on, and `left` of what has the digits so far are wanted
        const auto key_of = [](float v, int32_t c) { return (uint64_t)ordered(v) << 24 | (0xFFFFFFu - (uint32_t)c); };
        int32_t *bins = reinterpret_cast<int32_t *>(found);
        uint64_t key = 0;
        int32_t left = a.k;
        for (int shift = 48; shift >= 0 && n > kRoom; shift -= 8) {
            __syncthreads();
            for (int i = threadIdx.x; i < 256; i += THREADS) bins[i] = 0;
            __syncthreads();
            // equal digits follow each other in such rows, and are added once
            int32_t digit = 0, length = 0;
            z.again().each(none, [&](const Eight &v, int32_t c, uint32_t) {
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const uint64_t one = key_of(v.v[i], c + i);
                    if (one >> 24 == 0 || one >> (shift + 8) != key >> (shift + 8)) continue;
                    const int32_t next = (int32_t)(one >> shift & 255);
                    if (next != digit) {
                        if (length) atomicAdd(&bins[digit], length);
                        digit = next, length = 0;
                    }
                    length++;
                }
            });
            if (length) atomicAdd(&bins[digit], length);
            __syncthreads();
            // four digits a lane, the highest first: how many have its or a higher one
            int32_t of[4], sum = 0;
#pragma unroll
            for (int i = 0; i < 4; i++) of[i] = bins[255 - (lane * 4 + i)], sum += of[i];
            const int32_t all = wave_scan(sum);
            const int from = __builtin_ctzll(__ballot(all >= left));      // (as many as are wanted there are)
            int32_t above = __builtin_amdgcn_readlane(all - sum, from);
            int at = 0;
#pragma unroll
            for (int i = 0; i < 3; i++) {
                const int32_t more = __builtin_amdgcn_readlane(of[i], from);
                if (at == i && above + more < left) above += more, at++;
            }
            key |= (uint64_t)(255 - (from * 4 + at)) << shift;
            int32_t same = 0;
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (at == i) same = __builtin_amdgcn_readlane(of[i], from);
            n = a.k - left + above + same;
            left -= above;
        }
        __syncthreads();
        if (threadIdx.x == 0) used = 0;
        __syncthreads();
        z.again().each(none, [&](const Eight &v, int32_t c, uint32_t) {
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (v.v[i] > -INFINITY && key_of(v.v[i], c + i) >= key) put(v.v[i], c + i);
        });
        __syncthreads();
        n = used;
    }
    if constexpr (WAVES <= 4)
        if (n > kFew && n > 2 * a.k) {
            uint32_t values[kRoom / 64], least = 0;
#pragma unroll
            for (int i = 0; i < kRoom / 64; i++) values[i] = i * 64 + lane < n ? (uint32_t)(found[i * 64 + lane] >> 32) : 0u;
            for (int bit = 31; bit >= 0; bit--) {
                const uint32_t next = least | 1u << bit;
                int count = 0;
#pragma unroll
                for (int i = 0; i < kRoom / 64; i++)
                    if (i * 64 < n) count += __popcll(__ballot(values[i] >= next));
                if (count >= a.k) least = next;
            }
            uint64_t mine[kRoom / THREADS];
#pragma unroll
            for (int i = 0; i < kRoom / THREADS; i++) mine[i] = i * THREADS + (int)threadIdx.x < n ? found[i * THREADS + threadIdx.x] : 0u;
            __syncthreads();
            if (threadIdx.x == 0) used = 0;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kRoom / THREADS; i++)
                if (mine[i] && (uint32_t)(mine[i] >> 32) >= least) found[atomicAdd(&used, 1)] = mine[i];
            __syncthreads();
            n = used;
        }

    // places past the list's end are the lowest, up to whole groups of them that are read together
    constexpr int kTogether = 8;
    if ((int)threadIdx.x < kTogether) found[n + threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += THREADS) {
        const uint64_t mine = found[i];
        int rank = 0;
        for (int j = 0; j < n; j += kTogether) {
            uint64_t other[kTogether];
#pragma unroll
            for (int o = 0; o < kTogether; o++) other[o] = found[j + o];
#pragma unroll
            for (int o = 0; o < kTogether; o++) rank += other[o] > mine ? 1 : 0;
        }
        if (rank >= a.k) continue;
        a.index[row * a.k + rank] = (int32_t)(0xFFFFFFFFu - (uint32_t)mine);
        a.value[row * a.k + rank] = value_of((uint32_t)(mine >> 32));
        if (rank == a.k - 1) last = mine;
    }
    for (int i = n + threadIdx.x; i < a.k; i += THREADS) {
        a.index[row * a.k + i] = -1;
        a.value[row * a.k + i] = -INFINITY;
    }
    if (!a.rest) return;
    __syncthreads();
    // What is not listed is at most the last that is, which is what it is summed from.  All columns are, none as more than that last: the
    // k that are listed are then ones, and where half of the sum is left without them it has lost a bit.  Else the listed ones are left
    // out one by one: from the last listed still where the others come to more than two of it, from their own largest where they may be any
    // distance below it: a sum of packs has to have a one among them (PackSum), or others that lie 15 T and more below the last listed are rounded
    // away, all of them or some.  Such rows are gone through twice more (us, bf16, 4096 x 50021, k = 64: 140 where the sum is
    // left, 227 from the last listed, 259 from the others' largest; 512 x 130000 fp32, read again each time: 80 and 156).
    const uint64_t kth = last;
    const float least = kth ? value_of((uint32_t)(kth >> 32)) : -INFINITY, scale = a.per_T * kLog2e;
    const int32_t column = kth ? (int32_t)(0xFFFFFFFFu - (uint32_t)kth) : -1;
    const auto not_listed = [&](float v, int32_t c) { return v > least || (v == least && c <= column) ? -INFINITY : v; };
    float from = fmaxf(least, kLowest), sum = 0.0f;
    const Powers powers(scale, from);
    const auto sum_of = [&](auto &row, auto term) {
        PackSum sum;
        row.each(none, [&](const Eight &v, int32_t c, uint32_t) {
            float e[8];
#pragma unroll
            for (int i = 0; i < 8; i++) e[i] = term(v.v[i], c + i);
            sum.add(((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7])));
        });
        return over.sum(sum);
    };
    bool lost = true, near = false;               // (the same for all threads)
    if (kth && !powers.far()) {
        // (a NaN is the smaller of two numbers here: one instruction, where a comparison and a choice are two)
        const float one = fmaf(least, scale, -powers.K);
        sum = sum_of(z, [&](float v, int32_t) { return __builtin_amdgcn_exp2f(__builtin_elementwise_minimum(fmaf(v, scale, -powers.K), one)); });
        const float listed = (float)a.k * powers(least);
        lost = sum - listed < listed;
        sum = (sum - listed) * powers.lost();
        near = sum >= 2.0f;
    }
    if (lost) {
        auto again = z.again();
        if (!near) {
            float own_most = -INFINITY;
            z.each(none, [&](const Eight &v, int32_t c, uint32_t) {
#pragma unroll
                for (int i = 0; i < 8; i++) own_most = fmaxf(own_most, not_listed(v.v[i], c + i));
            });
            from = fmaxf(over.most(own_most), kLowest);
        }
        sum = sum_of(again, [&](float v, int32_t c) {
            const float other = not_listed(v, c);             // (an infinity like `from` is one too)
            return other == from ? 1.0f : __builtin_amdgcn_exp2f((other - from) * scale);
        });
    }
    if (threadIdx.x == 0) a.rest[row] = from * a.per_T + logf(sum);
}

// launch(wavefronts of a row, packs of eight that a lane holds).  Many rows go by as few wavefronts as hold them, which have fewer barriers and
// rounds over LDS to share (us, bf16, k = 32; 16384 x 1000 by 1 wavefront of 2 packs 20.8, by 2 of 1 33.8; x 2000 by 1 of 4 32.2, by 4 of 2
// 58.7; 15625 x 16000 by 4 of 8 132, by 8 of 4 144; 4997 x 50021 by 8 of 16 180, by 16 of 8 275, read again and again 237), a few rows by as
// many as shorten their way (128 x 2000 7.9, 5.8; x 16000 9.5, 8.2; x 64000 15.3, 14.0).  Of one wavefront's 64 largest values, or two's 128, a
// bound for many is too low (8192 x 2000, k = 64: 37 by one, 29 by four; x 4000, k = 128: 85 by two, 54 by four).  Of rows of up
// to 1024 columns that is not measured (8192 x 1000 by one wavefront: k = 64 28, 65 34, 128 42).  fp32 rows of more than 65536 columns are not held (1923 x 130000 335, held 551).
template <class T, class F>
int by_columns(int64_t columns, int64_t rows, int k, F launch)
{
    using std::integral_constant;
    const int64_t packs = (columns + 7) / 8;
    const bool few = rows <= 256;
    if (packs <= 64) return launch(integral_constant<int, 1>(), integral_constant<int, 1>());
    if (packs <= 128) return launch(integral_constant<int, 1>(), integral_constant<int, 2>());
    if (packs <= 256 && !few && k <= 48) return launch(integral_constant<int, 1>(), integral_constant<int, 4>());
    if (packs <= 512) return few || k > 96 ? launch(integral_constant<int, 4>(), integral_constant<int, 2>()) : launch(integral_constant<int, 2>(), integral_constant<int, 4>());
    if (packs <= 1024) return launch(integral_constant<int, 4>(), integral_constant<int, 4>());
    if (packs <= 2048) return few ? launch(integral_constant<int, 8>(), integral_constant<int, 4>()) : launch(integral_constant<int, 4>(), integral_constant<int, 8>());
    if (packs <= 4096) return few ? launch(integral_constant<int, 16>(), integral_constant<int, 4>()) : launch(integral_constant<int, 8>(), integral_constant<int, 8>());
    if (packs <= 8192) return few || T::planes == 3 ? launch(integral_constant<int, 16>(), integral_constant<int, 8>()) : launch(integral_constant<int, 8>(), integral_constant<int, T::planes == 1 ? 16 : 8>());
    if constexpr (T::planes == 1)
        if (packs <= 16384) return launch(integral_constant<int, 16>(), integral_constant<int, 16>());
    return launch(integral_constant<int, 16>(), integral_constant<int, 0>());
}

template <class T>
int run_top(const TopArgs &a, int64_t rows, hipStream_t st)
{
    return by_columns<T>(a.columns, rows, a.k, [&](auto waves, auto packs) -> int {
        constexpr int W = decltype(waves)::value, P = decltype(packs)::value;
        if (!fits_launch((uint64_t)rows * 64 * W)) return CCDC_ESIZE;
        k_top<T, W, P><<<(uint32_t)rows, 64 * W, 0, st>>>(a);
        return launched();
    });
}

}  // namespace

extern "C" {

int ccdc_top(const ccdc_block_t *b, int64_t rows, int64_t columns, const void *z, int64_t ldz, int k, double temperature, int32_t *index,
             float *value, float *rest, void *stream)
{
    const int rc = ready(b);
    if (rc != CCDC_OK) return rc;
    if (rows < 0 || columns < 1 || ldz < columns || k < 1 || k > kMostListed) return CCDC_EINVAL;
    const float heat = (float)temperature, per_T = 1.0f / heat;
    if (!(heat > 0.0f) || !std::isfinite(heat) || !std::isfinite(per_T * kLog2e)) return CCDC_EINVAL;
    if (rows == 0) return CCDC_OK;
    if (!fits(b, z) || !index || !value) return CCDC_EINVAL;
    for (const void *p : {(const void *)index, (const void *)value, (const void *)rest})
        if (!aligned(p, 4)) return CCDC_EINVAL;
    if (columns > kMostColumns) return CCDC_ESIZE;
    const TopArgs a{z, index, value, rest, ldz, (int32_t)columns, k, per_T};
    CCDC_BY_ELEM(b, (run_top<T>(a, rows, (hipStream_t)stream)));
}

}  // extern "C"
