// What the kernels over rows of logits share: a row by one workgroup, held in registers or read again, and sums over its threads.
#pragma once

#include "eight.hpp"

namespace ccdc {

constexpr int kMostListed = 128;              // of a row's top logits
constexpr float kLowest = -3.402823466e38f;   // stands in for -infinity as what is subtracted: exp(-infinity - kLowest) is 0

// The largest over a wavefront, the same for all its lanes.  (Lanes that nothing is moved to keep what they have.)
__device__ __forceinline__ float wave_most(float v)
{
    const auto moved = [](float x, auto control, auto rows) {
        return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(x), __float_as_int(x), decltype(control)::value, decltype(rows)::value, 15, false));
    };
    using std::integral_constant;
    v = fmaxf(v, moved(v, integral_constant<int, 0x111>(), integral_constant<int, 15>()));
    v = fmaxf(v, moved(v, integral_constant<int, 0x112>(), integral_constant<int, 15>()));
    v = fmaxf(v, moved(v, integral_constant<int, 0x114>(), integral_constant<int, 15>()));
    v = fmaxf(v, moved(v, integral_constant<int, 0x118>(), integral_constant<int, 15>()));
    v = fmaxf(v, moved(v, integral_constant<int, 0x142>(), integral_constant<int, 10>()));
    v = fmaxf(v, moved(v, integral_constant<int, 0x143>(), integral_constant<int, 12>()));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// The sum of a lane's and all lanes' before it.
__device__ __forceinline__ int32_t wave_scan(int32_t v)
{
    const auto moved = [](int32_t x, auto control, auto rows) {
        return __builtin_amdgcn_update_dpp(0, x, decltype(control)::value, decltype(rows)::value, 15, true);
    };
    using std::integral_constant;
    v += moved(v, integral_constant<int, 0x111>(), integral_constant<int, 15>());
    v += moved(v, integral_constant<int, 0x112>(), integral_constant<int, 15>());
    v += moved(v, integral_constant<int, 0x114>(), integral_constant<int, 15>());
    v += moved(v, integral_constant<int, 0x118>(), integral_constant<int, 15>());
    v += moved(v, integral_constant<int, 0x142>(), integral_constant<int, 10>());
    return v + moved(v, integral_constant<int, 0x143>(), integral_constant<int, 12>());
}

// exp((v - from) / T) as a power of two, in one product and sum: 2^(v scale - K) with K = from scale rounded.  What K is off by is
// exact as a product and sum again, below one while K is below 2^24, and `lost` undoes it in a sum of these.  Rows further from zero
// (those of which the lowest number of the type is the largest, say) are `far`: there the difference is taken first.
struct Powers {
    float scale, from, K;
    __device__ __forceinline__ Powers(float scale, float from) : scale(scale), from(from), K(from * scale) {}
    __device__ __forceinline__ bool far() const { return !(fabsf(K) < 16777216.0f); }
    __device__ __forceinline__ float operator()(float v) const { return __builtin_amdgcn_exp2f(fmaf(v, scale, -K)); }
    __device__ __forceinline__ float lost() const { return __builtin_amdgcn_exp2f(-fmaf(from, scale, -K)); }
    __device__ __forceinline__ float difference(float v) const { return __builtin_amdgcn_exp2f((v - from) * scale); }
};

// As wave_sum of 32 bits (element.hpp).
__device__ __forceinline__ double wave_sum(double v)
{
    const auto moved = [](double x, auto control, auto rows) {
        const int2 from = __builtin_bit_cast(int2, x);
        int2 to;
        to.x = __builtin_amdgcn_update_dpp(0, from.x, decltype(control)::value, decltype(rows)::value, 15, true);
        to.y = __builtin_amdgcn_update_dpp(0, from.y, decltype(control)::value, decltype(rows)::value, 15, true);
        return __builtin_bit_cast(double, to);
    };
    using std::integral_constant;
    v += moved(v, integral_constant<int, 0x111>(), integral_constant<int, 15>());
    v += moved(v, integral_constant<int, 0x112>(), integral_constant<int, 15>());
    v += moved(v, integral_constant<int, 0x114>(), integral_constant<int, 15>());
    v += moved(v, integral_constant<int, 0x118>(), integral_constant<int, 15>());
    v += moved(v, integral_constant<int, 0x142>(), integral_constant<int, 10>());
    v += moved(v, integral_constant<int, 0x143>(), integral_constant<int, 12>());
    const int2 all = __builtin_bit_cast(int2, v);
    return __builtin_bit_cast(double, int2{__builtin_amdgcn_readlane(all.x, 63), __builtin_amdgcn_readlane(all.y, 63)});
}

// A sum of the packs of a row that is the same whatever thread has which of them: in 64 bits, of numbers rounded to 2^-32, which is exact
// up to 2^21 (a pack is at most 8 exponentials of at most 2^(1/2), of 2^17 packs).  The roundings are 2^-33 a pack, of a sum that has to be
// one or so at least (2^(-1/2)): whoever sums takes exponentials from the largest of what is summed, or knows of as much.  Four
// instructions a pack of eight.
struct PackSum {
    double sum = 0.0;
    __device__ __forceinline__ void add(float pack)
    {
        constexpr double kRound = 1.5 * 1048576.0;            // numbers from 2^20 to 2^21 are whole 2^-32
        sum += ((double)pack + kRound) - kRound;
    }
};

// Sums and largest values over a row's threads, wavefronts by LDS in their order.  Parts of the LDS in turn, so that one barrier is
// enough: who writes a part again has met the others since they read it.
template <int WAVES>
struct OverRow {
    double *part;                                 // [2][WAVES]
    int at = 0;

    template <class V, class F>
    __device__ __forceinline__ V join(V v, F both)
    {
        if constexpr (WAVES == 1) return v;
        double *slot = part + at;
        at = WAVES - at;
        if (threadIdx.x % 64 == 0) slot[threadIdx.x / 64] = v;
        __syncthreads();
        v = (V)slot[0];
#pragma unroll
        for (int i = 1; i < WAVES; i++) v = both(v, (V)slot[i]);
        return v;
    }
    __device__ __forceinline__ float sum(float v)
    {
        return join(wave_sum(v), [](float a, float b) { return a + b; });
    }
    __device__ __forceinline__ float sum(const PackSum &s)
    {
        return (float)join(wave_sum(s.sum), [](double a, double b) { return a + b; });
    }
    __device__ __forceinline__ float most(float v)
    {
        return join(wave_most(v), [](float a, float b) { return fmaxf(a, b); });
    }
};

// Word w of a pack with -infinity where a bit is set (16-bit elements: two a word).
template <class T>
__device__ __forceinline__ uint32_t hide_word(uint32_t word, uint32_t bits, int w)
{
    if constexpr (sizeof(typename T::elem) == 4) {
        const uint32_t mask = (uint32_t)__builtin_amdgcn_sbfe((int)bits, w, 1);
        return (word & ~mask) | (0xFF800000u & mask);
    } else {
        constexpr uint32_t kNone = std::is_same<T, ElemF16>::value ? 0xFC00FC00u : 0xFF80FF80u;
        const uint32_t low = (uint32_t)__builtin_amdgcn_sbfe((int)bits, 2 * w, 1), high = (uint32_t)__builtin_amdgcn_sbfe((int)bits, 2 * w + 1, 1);
        const uint32_t mask = (low & 0xFFFFu) | (high & 0xFFFF0000u);
        return (word & ~mask) | (kNone & mask);
    }
}

// A row in packs of eight columns.  The last is read as the row's last eight, and what the one before has too is hidden: every read
// is of eight columns in the row, also those of lanes past its end, and none takes a way of its own.
// A thread has packs (its place) + i * (threads): the first PACKS held in registers as loaded, LDS more in LDS, and, where the row is longer
// (REST), any number that are read whenever they are asked for.  What is hidden is -infinity.
template <class T, int WAVES, int PACKS, int LDS = 0, bool REST = PACKS == 0>
struct Row {
    using E = typename T::elem;
    static constexpr int kThreads = 64 * WAVES, kWords = 2 * sizeof(E), HELD = PACKS + LDS;
    static_assert(LDS == 0 || kWords == 4);
    const E *p;
    int32_t columns;
    uint32_t held[PACKS ? PACKS : 1][kWords];
    Bytes16 *room;                        // the thread's first pack in LDS

    __device__ __forceinline__ void get(int i, uint32_t (&words)[kWords]) const
    {
        if (i < PACKS) {
#pragma unroll
            for (int w = 0; w < kWords; w++) words[w] = held[i < PACKS ? i : 0][w];
        } else {
            __builtin_memcpy(words, &room[(i - PACKS) * kThreads], 16);
        }
    }
    __device__ __forceinline__ void set(int i, const uint32_t (&words)[kWords])
    {
        if (i < PACKS) {
#pragma unroll
            for (int w = 0; w < kWords; w++) held[i < PACKS ? i : 0][w] = words[w];
        } else {
            __builtin_memcpy(&room[(i - PACKS) * kThreads], words, 16);
        }
    }
    struct Pack8 {
        int32_t start;                    // first column that is read
        uint32_t valid;                   // of the eight: those that are this pack's
    };
    __device__ __forceinline__ Pack8 pack_of(int32_t j) const
    {
        const int32_t first = j * 8, start = max(min(first, columns - 8), 0), from = first - start;
        return {start, from < 8 ? (1u << min(columns - start, 8)) - (1u << from) : 0u};
    }
    __device__ __forceinline__ void read(uint32_t (&words)[kWords], int32_t start) const
    {
        if (columns >= 8) {               // (the same for all)
            constexpr int W = 16 / sizeof(E);
            using P = Pack<E, W>;
#pragma unroll
            for (int h = 0; h < 8 / W; h++) {
                const P q = load_pack_any<true, P, E>(p + start + h * W);
                __builtin_memcpy(&words[h * 4], &q, sizeof q);
            }
        } else {
            const Raw8<T> raw = load_raw<T>(p, columns);
            __builtin_memcpy(words, &raw, sizeof raw);
        }
    }
    // Whether any thread's pack i is in the row.
    __device__ __forceinline__ bool some(int i) const { return i * kThreads * 8 < columns; }
    // Not held, for what few rows need: the same row read again.
    __device__ __forceinline__ Row<T, WAVES, 0> again() const
    {
        Row<T, WAVES, 0> row;
        row.p = p, row.columns = columns;
        return row;
    }
    __device__ __forceinline__ void load(const void *base, int64_t at, int32_t of)
    {
        p = (const E *)base + at;
        columns = of;
#pragma unroll
        for (int i = 0; i < PACKS; i++)
            if (some(i)) read(held[i], pack_of(fresh((int32_t)threadIdx.x + i * kThreads)).start);
        if constexpr (LDS > 0) {
            uint32_t words[LDS][kWords];
#pragma unroll
            for (int i = 0; i < LDS; i++)
                if (some(PACKS + i)) read(words[i], pack_of(fresh((int32_t)threadIdx.x + (PACKS + i) * kThreads)).start);
#pragma unroll
            for (int i = 0; i < LDS; i++)
                if (some(PACKS + i)) set(PACKS + i, words[i]);
        }
    }
    // Eight numbers, widened.  The compiler does not see that a held pack is what it was in another pass, or it would keep all 16-bit
    // numbers widened.
    __device__ __forceinline__ static Eight wide(const uint32_t (&from)[kWords], uint32_t shift, uint32_t mask)
    {
        Eight v;
        if constexpr (std::is_same<T, ElemBF16>::value) {
#pragma unroll
            for (int w = 0; w < 4; w++) v.v[2 * w] = __uint_as_float(from[w] << shift), v.v[2 * w + 1] = __uint_as_float(from[w] & mask);
        } else {
            uint32_t words[kWords];
#pragma unroll
            for (int w = 0; w < kWords; w++) {
                words[w] = from[w];
                if (T::planes == 1) asm volatile("" : "+v"(words[w]));
            }
            Raw8<T> raw;
            __builtin_memcpy(&raw, words, sizeof raw);
            v = widen(raw);
        }
        return v;
    }
    // Registers of whole words from here on, whatever ways lead here.
    __device__ __forceinline__ void whole()
    {
#pragma unroll
        for (int i = 0; i < PACKS; i++)
#pragma unroll
            for (int w = 0; w < kWords; w++) asm volatile("" : "+v"(held[i][w]));
    }
    // Hides the columns of held packs that hidden(first of eight columns) has bits of, and f(values) for each pack.  END: only what is past the
    // row's end is hidden, of the packs there.
    template <bool END, class H, class F>
    __device__ __forceinline__ void hide_held(H hidden, F f)
    {
        const uint32_t shift = fresh_uniform(16u), mask = fresh_uniform(0xFFFF0000u);
        whole();
#pragma unroll
        for (int i = 0; i < HELD; i++) {
            if (!some(i) || (END && (i + 1) * kThreads * 8 <= columns)) continue;
            const Pack8 pack = pack_of(fresh((int32_t)threadIdx.x + i * kThreads));
            const uint32_t bits = (hidden(pack.start) | ~pack.valid) & 0xFFu;
            uint32_t words[kWords];
            get(i, words);
#pragma unroll
            for (int w = 0; w < kWords; w++) words[w] = hide_word<T>(words[w], bits, w);
            set(i, words);
            if constexpr (!END) f(wide(words, shift, mask));
        }
        whole();
        if constexpr (END)
#pragma unroll
            for (int i = 0; i < HELD; i++) {
                if (!some(i)) continue;
                uint32_t words[kWords];
                get(i, words);
                f(wide(words, shift, mask));
            }
    }
    // f(values, first of their eight columns, which of them are this pack's) for each pack; those that are read now are hidden now.
    template <class H, class F>
    __device__ __forceinline__ void each(H hidden, F f)
    {
        const uint32_t shift = fresh_uniform(16u), mask = fresh_uniform(0xFFFF0000u);
#pragma unroll
        for (int i = 0; i < HELD; i++) {
            if (!some(i)) continue;
            const Pack8 pack = pack_of(fresh((int32_t)threadIdx.x + i * kThreads));
            uint32_t words[kWords];
            get(i, words);
            f(wide(words, shift, mask), pack.start, pack.valid);
            // one after the other: with packs interleaved a row of eight takes half as many registers again
            __builtin_amdgcn_sched_barrier(0);
        }
        rest(hidden, f);
    }
    // Of those that are not held.
    template <class H, class F>
    __device__ __forceinline__ void rest(H hidden, F f)
    {
        if constexpr (!REST) return;
        const uint32_t shift = fresh_uniform(16u), mask = fresh_uniform(0xFFFF0000u);
        // two packs on their way at a time
        const int32_t packs = (columns + 7) / 8;
        for (int32_t j = (int32_t)threadIdx.x + HELD * kThreads; j < packs; j += 2 * kThreads) {
            const Pack8 pack[2] = {pack_of(j), pack_of(j + kThreads)};
            uint32_t words[2][kWords];
#pragma unroll
            for (int h = 0; h < 2; h++) read(words[h], pack[h].start);
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const uint32_t bits = (hidden(pack[h].start) | ~pack[h].valid) & 0xFFu;
                if (bits)                 // few packs
#pragma unroll
                    for (int w = 0; w < kWords; w++) words[h][w] = hide_word<T>(words[h][w], bits, w);
                if (pack[h].valid) f(wide(words[h], shift, mask), pack[h].start, pack[h].valid);
            }
        }
    }
    // Writes eight columns from `start` on, those that are valid.  Rows that are read again go past the caches, which have then more of
    // what is read (1500 x 131071 f16 250 -> 233 us).
    static __device__ __forceinline__ void store(E *to, const Eight &v, uint32_t valid)
    {
        if (valid == 0xFFu && REST) {
            constexpr int W = 16 / sizeof(E);
            using P = Pack<E, W>;
#pragma unroll
            for (int h = 0; h < 8 / W; h++) {
                P q;
#pragma unroll
                for (int i = 0; i < W; i++) q.v[i] = narrow<T>(v.v[h * W + i]);
                store_stream_any<P, E>(to + h * W, q);
            }
        } else if (valid == 0xFFu) {
            store_eight<T>(to, v, 8);
        } else {
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (valid >> e & 1) to[e] = narrow<T>(v.v[e]);
        }
    }
};

}  // namespace ccdc
