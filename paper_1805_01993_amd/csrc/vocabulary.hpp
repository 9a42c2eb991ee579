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

// Sums and largest values over a row's threads, wavefronts by LDS in their order.  Parts of the LDS in turn, so that one barrier is
// enough: who writes a part again has met the others since they read it.
template <int WAVES>
struct OverRow {
    float *part;                                  // [2][WAVES]
    int at = 0;

    template <class F>
    __device__ __forceinline__ float join(float v, F both)
    {
        if constexpr (WAVES == 1) return v;
        float *slot = part + at;
        at = WAVES - at;
        if (threadIdx.x % 64 == 0) slot[threadIdx.x / 64] = v;
        __syncthreads();
        v = slot[0];
#pragma unroll
        for (int i = 1; i < WAVES; i++) v = both(v, slot[i]);
        return v;
    }
    __device__ __forceinline__ float sum(float v)
    {
        return join(wave_sum(v), [](float a, float b) { return a + b; });
    }
    __device__ __forceinline__ float most(float v)
    {
        return join(wave_most(v), [](float a, float b) { return fmaxf(a, b); });
    }
};

// The bits of a pack's columns that are past the row's end, `left` columns on.
__device__ __forceinline__ uint32_t past(int32_t left) { return left >= 8 ? 0u : 0xFFu << max(left, 0) & 0xFFu; }

// A pack with -infinity where a bit is set.
template <class T>
__device__ __forceinline__ Raw8<T> hide(Raw8<T> raw, uint32_t bits)
{
    using E = typename T::elem;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        if constexpr (sizeof(E) == 4) raw.p.v[i] = bits >> i & 1 ? -INFINITY : raw.p.v[i];
        else raw.p.v[i] = bits >> i & 1 ? (E)(std::is_same<T, ElemF16>::value ? 0xFC00 : 0xFF80) : raw.p.v[i];
    }
    return raw;
}

// The packs of eight columns that a thread has of a row: (its place) + i * (threads).  PACKS > 0: as many at the most, held in registers as
// loaded; 0: any number, read whenever they are asked for.  What is hidden, and what is past the row's end, is -infinity.
template <class T, int WAVES, int PACKS>
struct Row {
    using E = typename T::elem;
    static constexpr int kThreads = 64 * WAVES, kWords = 2 * sizeof(E);
    const E *p;
    int32_t columns;
    uint32_t held[PACKS ? PACKS : 1][kWords];

    __device__ __forceinline__ void load(const void *base, int64_t at, int32_t of)
    {
        p = (const E *)base + at;
        columns = of;
#pragma unroll
        for (int i = 0; i < PACKS; i++) {
            const int32_t c = fresh((int32_t)threadIdx.x + i * kThreads) * 8;
            Raw8<T> raw = {};
            if (c < columns) raw = load_raw<T>(p + c, columns - c);
            __builtin_memcpy(held[i], &raw, sizeof raw);
        }
    }
    // Pack i as held; the compiler sees another number each time, or it would keep all packs widened from one pass to the next.
    __device__ __forceinline__ Raw8<T> pack(int i)
    {
#pragma unroll
        for (int w = 0; w < kWords; w++) asm volatile("" : "+v"(held[i][w]));
        Raw8<T> raw;
        __builtin_memcpy(&raw, held[i], sizeof raw);
        return raw;
    }
    // Hides the columns that hidden(first column of a pack) has bits of.
    template <class H>
    __device__ __forceinline__ void hide_held(H hidden)
    {
#pragma unroll
        for (int i = 0; i < PACKS; i++) {
            const int32_t c = fresh((int32_t)threadIdx.x + i * kThreads) * 8;
            const Raw8<T> raw = hide<T>(pack(i), c < columns ? hidden(c) | past(columns - c) : 0xFFu);
            __builtin_memcpy(held[i], &raw, sizeof raw);
        }
    }
    // f(values, first column, columns of them in the row, which may be none) for each pack.
    template <class H, class F>
    __device__ __forceinline__ void each(H hidden, F f)
    {
        if constexpr (PACKS > 0) {
#pragma unroll
            for (int i = 0; i < PACKS; i++) {
                const int32_t c = fresh((int32_t)threadIdx.x + i * kThreads) * 8;
                f(widen(pack(i)), c, columns - c);
            }
        } else {
            // two packs on their way at a time
            for (int32_t c = (int32_t)threadIdx.x * 8; c < columns; c += 2 * kThreads * 8) {
                const int32_t next = c + kThreads * 8;
                const Raw8<T> one = load_raw<T>(p + c, columns - c);
                const Raw8<T> two = next < columns ? load_raw<T>(p + next, columns - next) : Raw8<T>{};
                f(widen(hide<T>(one, hidden(c) | past(columns - c))), c, columns - c);
                if (next < columns) f(widen(hide<T>(two, hidden(next) | past(columns - next))), next, columns - next);
            }
        }
    }
};

// Wavefronts of a row and packs that a lane holds of it: launch(waves, packs), packs 0 where the row is more than the registers hold.  Rows
// of 1024 threads have 128 registers a lane; two such workgroups are on a CU up to four packs, so that one's loads meet the other's
// sums.
template <class T, class F>
int by_columns(int64_t columns, F launch)
{
    using std::integral_constant;
    const int64_t packs = (columns + 7) / 8;
    if (packs <= 64) return launch(integral_constant<int, 1>(), integral_constant<int, 1>());
    if (packs <= 128) return launch(integral_constant<int, 2>(), integral_constant<int, 1>());
    if (packs <= 512) return launch(integral_constant<int, 4>(), integral_constant<int, 2>());
    if (packs <= 1024) return launch(integral_constant<int, 4>(), integral_constant<int, 4>());
    if (packs <= 2048) return launch(integral_constant<int, 8>(), integral_constant<int, 4>());
    if (packs <= 4096) return launch(integral_constant<int, 16>(), integral_constant<int, 4>());
    if (packs <= 8192) return launch(integral_constant<int, 16>(), integral_constant<int, 8>());
    return launch(integral_constant<int, 16>(), integral_constant<int, 0>());
}

}  // namespace ccdc
