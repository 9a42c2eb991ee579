// What the kernels of a trained block use of the device, on the host (test infrastructure only; included in front of every translated
// source).  A lane is a fibre: the lanes of a workgroup run one after the other up to where the kernel meets (a barrier, an
// exchange within the wavefront), always in the same order, so a barrier that is missing shows as a wrong value every time.  An
// exchange is of all 64 lanes of a wavefront but those that have returned; one that not all others come to stops the run.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

namespace shim {
typedef short Bits4 __attribute__((ext_vector_type(4)));
typedef float Acc4 __attribute__((ext_vector_type(4)));
typedef float Acc16 __attribute__((ext_vector_type(16)));

extern int force;                                     // which tile: -1 as the library's rules say, 1 large, 2 small, 0 small with more of it in LDS
extern thread_local unsigned char *lds;               // byte 0 of the workgroup's LDS, as copy_to_lds has it

void *block_shared(size_t bytes, size_t align);       // the running workgroup's next __shared__ array: a block of its own
void wave_in_step();                                  // every lane of the wavefront has come here
uint32_t read_lane(uint32_t v, int lane);
uint32_t update_dpp(uint32_t old, uint32_t v, int control, int rows, int banks, bool bound);
// 16 bytes a lane, lane after lane from byte `to` on.  Arrives when it is waited for and no earlier: wait_copies leaves the last `but`.
void copy_to_lds(uint32_t to, const void *from);
void wait_copies(int but);
Bits4 read_transposed(const void *lane_address);
// C + A B' of a wavefront, 16 x 16 x 32 and 32 x 32 x 16; numbers of 16 bits as bits
void multiply16(const uint16_t *a, const uint16_t *b, bool bf, float *c);
void multiply32(const uint16_t *a, const uint16_t *b, bool bf, float *c);

template <class V, class C>
C multiply(const V &a, const V &b, C c, bool bf)
{
    static_assert(sizeof(V) == 16 && (sizeof(C) == 16 || sizeof(C) == 64));
    uint16_t x[8], y[8];
    float z[sizeof(C) / 4];
    __builtin_memcpy(x, &a, 16);
    __builtin_memcpy(y, &b, 16);
    __builtin_memcpy(z, &c, sizeof(C));
    if constexpr (sizeof(C) == 16) multiply16(x, y, bf, z);
    else multiply32(x, y, bf, z);
    __builtin_memcpy(&c, z, sizeof(C));
    return c;
}
}  // namespace shim

inline int __float_as_int(float f) { int v; __builtin_memcpy(&v, &f, 4); return v; }
inline float __int_as_float(int v) { float f; __builtin_memcpy(&f, &v, 4); return f; }
inline float __expf(float x) { return std::exp(x); }
template <class A, class B>
inline std::common_type_t<A, B> min(A a, B b) { return (std::common_type_t<A, B>)b < (std::common_type_t<A, B>)a ? b : a; }
template <class A, class B>
inline std::common_type_t<A, B> max(A a, B b) { return (std::common_type_t<A, B>)a < (std::common_type_t<A, B>)b ? b : a; }

#define __builtin_amdgcn_readfirstlane(v) (v)         // (asked for of what is one for a wavefront only)
#define __builtin_amdgcn_readlane(v, l) ((int)shim::read_lane((uint32_t)(v), l))
#define __builtin_amdgcn_update_dpp(o, v, c, r, k, b) ((int)shim::update_dpp((uint32_t)(o), (uint32_t)(v), c, r, k, b))
#define __builtin_amdgcn_sched_barrier(m) ((void)0)
#define __builtin_amdgcn_s_setprio(p) ((void)0)
#define __builtin_amdgcn_ds_read_tr16_b64_v4i16(p) shim::read_transposed(p)
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, x, y, z) shim::multiply(a, b, c, true)
#define __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, x, y, z) shim::multiply(a, b, c, false)
#define __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, x, y, z) shim::multiply(a, b, c, true)
#define __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, x, y, z) shim::multiply(a, b, c, false)
