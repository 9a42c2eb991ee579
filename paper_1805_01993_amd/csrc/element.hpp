// What the kernels of a block share: element types, eight elements of a row at a time, dropout.
#pragma once

#include "block.hpp"
#include "common.hpp"

namespace ccdc {

struct ElemF32 : HybF32 {
    static constexpr int planes = 3;
};
struct ElemBF16 : HybBF16 {
    static constexpr int planes = 1;
};
struct ElemF16 : HybF16 {
    static constexpr int planes = 1;
};

// Eight consecutive elements of a row, widened: 16 bytes of a 16-bit format, the unit of its loads and stores, and the
// elements that one call of the generator decides on.  Rows are aligned to their elements only (global memory serves
// unaligned packs); the last pack of a row that is no whole number of packs is moved element by element.
struct Eight {
    float v[8];
};

// The same number, as one that the compiler has not seen: comparisons with it are made where they are used.  Kept from one pack to
// the next they are 64-bit masks in scalar registers, more than there are.
__device__ __forceinline__ int fresh(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// The same for numbers and addresses that are one for all lanes.
template <class V>
__device__ __forceinline__ V fresh_uniform(V v)
{
    asm volatile("" : "+s"(v));
    return v;
}

// 1 for the first `valid` of a pack's elements, else 0, without a mask.
__device__ __forceinline__ int inside(int valid, int i) { return min(max(valid - i, 0), 1); }

// Rounded to nearest even.  Unlike a payload's sums (Hyb16::narrow) a NaN keeps what the conversion makes of it: two instructions an
// element less.
template <class T>
__device__ __forceinline__ typename T::elem narrow(float x)
{
    if constexpr (sizeof(typename T::elem) == 2) {
        typename T::elem out;
        if constexpr (std::is_base_of<HybBF16, T>::value) {
            const __bf16 h = (__bf16)x;
            __builtin_memcpy(&out, &h, 2);
        } else {
            const _Float16 h = (_Float16)x;
            __builtin_memcpy(&out, &h, 2);
        }
        return out;
    } else {
        return x;
    }
}

// As loaded; zeros past the row's end.
template <class T>
struct Raw8 {
    Pack<typename T::elem, 8> p;
};

template <class T>
__device__ __forceinline__ Raw8<T> load_raw(const typename T::elem *p, int valid)
{
    using E = typename T::elem;
    constexpr int W = 16 / sizeof(E);
    using P = Pack<E, W>;
    Raw8<T> out;
    valid = fresh(valid);
    if (valid >= 8) {
#pragma unroll
        for (int h = 0; h < 8 / W; h++) {
            const P q = load_pack_any<true, P, E>(p + h * W);
#pragma unroll
            for (int i = 0; i < W; i++) out.p.v[h * W + i] = q.v[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const E e = p[min(i, valid - 1)];
            if constexpr (sizeof(E) == 2) out.p.v[i] = (E)(e & -inside(valid, i));
            else out.p.v[i] = __int_as_float(__float_as_int(e) & -inside(valid, i));
        }
    }
    return out;
}

template <class T>
__device__ __forceinline__ Eight widen(const Raw8<T> &raw)
{
    Eight out;
#pragma unroll
    for (int i = 0; i < 8; i++) out.v[i] = T::widen(raw.p.v[i]);
    return out;
}

template <class T>
__device__ __forceinline__ Eight load_eight(const typename T::elem *p, int valid)
{
    return widen(load_raw<T>(p, valid));
}

template <class T>
__device__ __forceinline__ void store_eight(typename T::elem *p, const Eight &x, int valid)
{
    using E = typename T::elem;
    constexpr int W = 16 / sizeof(E);
    using P = Pack<E, W>;
    valid = fresh(valid);
    if (valid >= 8) {
#pragma unroll
        for (int h = 0; h < 8 / W; h++) {
            P q;
#pragma unroll
            for (int i = 0; i < W; i++) q.v[i] = narrow<T>(x.v[h * W + i]);
            store_any<P, E>(p + h * W, q);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < valid) p[i] = narrow<T>(x.v[i]);
    }
}

// Dropout (ccdc.h): Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011).  Eight
// 16-bit numbers a call decide on eight neighbours of a row: a call's twenty 32 x 32 bit products are what dropout
// computes, so half the bits a decision are half of that, for a probability that is a multiple of 2^-16.
struct Dropout {
    uint32_t key[2], site, threshold;
    float scale;
};

inline Dropout make_dropout(double p, uint32_t site, uint64_t seed)
{
    const uint32_t t = dropout_threshold(p);
    return {{(uint32_t)seed, (uint32_t)(seed >> 32)}, site, t, t >= 65536 ? 0.0f : 65536.0f / (float)(65536 - t)};
}

// The random numbers of columns 8 * unit .. 8 * unit + 7 of a row, two a word.
struct Words {
    uint32_t w[4];
};
__device__ __forceinline__ Words dropout_words(const Dropout &d, uint32_t id, uint32_t token, uint32_t unit)
{
    uint32_t c0 = unit, c1 = token, c2 = id, c3 = d.site, k0 = d.key[0], k1 = d.key[1];
#pragma unroll
    for (int round = 0; round < 10; round++) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}
__device__ __forceinline__ uint32_t half_of(const Words &r, int i) { return i % 2 ? r.w[i / 2] >> 16 : r.w[i / 2] & 0xFFFFu; }

// Takes out of eight values what dropout takes out (an infinity or no number too), and multiplies the others.
__device__ __forceinline__ void drop_eight(Eight &v, const Dropout &d, uint32_t id, uint32_t token, uint32_t unit)
{
    const Words r = dropout_words(d, id, token, unit);
#pragma unroll
    for (int i = 0; i < 8; i++) v.v[i] = half_of(r, i) >= d.threshold ? v.v[i] * d.scale : 0.0f;
}

// The same as factors, 0 for what is taken out.
__device__ __forceinline__ Eight dropout_factors(const Dropout &d, uint32_t id, uint32_t token, uint32_t unit)
{
    const Words r = dropout_words(d, id, token, unit);
    Eight f;
#pragma unroll
    for (int i = 0; i < 8; i++) f.v[i] = half_of(r, i) >= d.threshold ? d.scale : 0.0f;
    return f;
}

// What is taken out counts for nothing, whatever it was (an infinity or no number too).
__device__ __forceinline__ float kept(float v, float factor) { return factor != 0.0f ? v * factor : 0.0f; }

inline int ready(const ccdc_block_t *b)
{
    if (!b) return CCDC_EINVAL;
    if (!b->uploaded) return CCDC_ESTATE;
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) {
        (void)hipGetLastError();
        return CCDC_EHIP;
    }
    return dev == b->device ? CCDC_OK : CCDC_ESTATE;
}

// Whether p may be a matrix of the block's elements (null: only where that is allowed).
inline bool fits(const ccdc_block_t *b, const void *p, bool null_too = false)
{
    return p ? aligned(p, (size_t)b->elem) : null_too;
}

}  // namespace ccdc

// Evaluates CALL with the block's element type as T, inside a function that has `using namespace ccdc`.
#define CCDC_BY_ELEM(b, CALL)                                                     \
    do {                                                                          \
        switch ((b)->c.mode) {                                                    \
        case CCDC_BF16_SUM_XOR: { using T = ElemBF16; return CALL; }              \
        case CCDC_F16_SUM_XOR: { using T = ElemF16; return CALL; }                \
        default: { using T = ElemF32; return CALL; }                              \
        }                                                                         \
    } while (0)
