// Device helpers of the 8-bit operators: rows of fp32 or bf16 at any byte address.
#pragma once

#include "nm_q8_internal.h"

namespace nm {

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// two fp32 as bf16, nearest even, a NaN stays one (one instruction on gfx950)
__device__ inline unsigned bf16_pair(float lo, float hi)
{
    return __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// Eight adjacent values, or one.  Through memcpy: global memory takes 16-byte accesses at any address.
template <bool BF16> struct Elem;
template <> struct Elem<false> {
    static constexpr int kBytes = 4;
    static __device__ inline void load8(const char* p, float (&v)[8])
    {
        u32x4 a, b;
        __builtin_memcpy(&a, p, 16);
        __builtin_memcpy(&b, p + 16, 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = __uint_as_float(a[i]); v[4 + i] = __uint_as_float(b[i]); }
    }
    static __device__ inline float load1(const char* p) { float f; __builtin_memcpy(&f, p, 4); return f; }
    static __device__ inline void store8(char* p, const float (&v)[8])
    {
        u32x4 a, b;
#pragma unroll
        for (int i = 0; i < 4; ++i) { a[i] = __float_as_uint(v[i]); b[i] = __float_as_uint(v[4 + i]); }
        __builtin_memcpy(p, &a, 16);
        __builtin_memcpy(p + 16, &b, 16);
    }
    static __device__ inline void store1(char* p, float f) { __builtin_memcpy(p, &f, 4); }
};
template <> struct Elem<true> {
    static constexpr int kBytes = 2;
    static __device__ inline void load8(const char* p, float (&v)[8])
    {
        u32x4 a;
        __builtin_memcpy(&a, p, 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(a[i] << 16); v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u); }
    }
    static __device__ inline float load1(const char* p) { unsigned short h; __builtin_memcpy(&h, p, 2); return __uint_as_float((unsigned)h << 16); }
    static __device__ inline void store8(char* p, const float (&v)[8])
    {
        u32x4 a;
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
        __builtin_memcpy(p, &a, 16);
    }
    static __device__ inline void store1(char* p, float f) { unsigned short h = (unsigned short)(bf16_pair(f, 0.0f) & 0xffffu); __builtin_memcpy(p, &h, 2); }
};

}  // namespace nm
