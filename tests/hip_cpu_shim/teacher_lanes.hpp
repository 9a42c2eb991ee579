// What the kernels that learn from a teacher use of the device besides (test infrastructure only; included after block_lanes.hpp).
#pragma once

#include "block_lanes.hpp"

namespace shim {
uint64_t ballot(bool v);
void copy_words_to_lds(uint32_t to, const void *from);
void multiply_eight16(const void *a, int scale_a, const void *b, int scale_b, float *c);
void multiply_eight32(const void *a, int scale_a, const void *b, int scale_b, float *c);
int to_eight(float v);
float of_eight(unsigned char bits);

template <class V, class C>
C multiply_eight(V a, V b, C c, int sa, int sb)
{
    float z[sizeof(C) / 4];
    __builtin_memcpy(z, &c, sizeof(C));
    if constexpr (sizeof(C) == 16) multiply_eight16(&a, sa, &b, sb, z);
    else multiply_eight32(&a, sa, &b, sb, z);
    __builtin_memcpy(&c, z, sizeof(C));
    return c;
}
typedef __bf16 Two __attribute__((ext_vector_type(2)));
inline Two widen_eight(int bits, float scale, bool high)
{
    const unsigned u = (unsigned)bits >> (high ? 16 : 0);
    return Two{(__bf16)(of_eight(u & 255) * scale), (__bf16)(of_eight(u >> 8 & 255) * scale)};
}
inline int narrow_eight(float a, float b, int old, bool high)
{
    const unsigned two = (unsigned)(to_eight(a) | to_eight(b) << 8);
    return (int)(high ? ((unsigned)old & 0xFFFFu) | two << 16 : ((unsigned)old & 0xFFFF0000u) | two);
}
}  // namespace shim

struct int2 {
    int x, y;
};
inline int atomicAdd(int *p, int v) { const int old = *p; *p += v; return old; }
inline uint32_t atomicOr(uint32_t *p, uint32_t v) { const uint32_t old = *p; *p |= v; return old; }
#define __ballot(v) shim::ballot(v)
#define __any(v) (shim::ballot(v) != 0)
#define __popcll(v) __builtin_popcountll(v)
#define __builtin_amdgcn_exp2f(x) std::exp2(x)
#define __builtin_amdgcn_sbfe(v, at, bits) (-(int)((unsigned)(v) >> (at) & 1u))        /* (asked for one bit) */
#define __builtin_amdgcn_cvt_pk_fp8_f32(a, b, old, high) shim::narrow_eight(a, b, old, high)
#define __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, scale, high) shim::widen_eight(v, scale, high)
#define __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, x, y, oa, sa, ob, sb) shim::multiply_eight(a, b, c, sa, sb)
#define __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, x, y, oa, sa, ob, sb) shim::multiply_eight(a, b, c, sa, sb)
