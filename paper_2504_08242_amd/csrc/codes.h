// 8-bit codes of a paged pool (include/jupiter_paged.h): what a code stands for, and the code nearest to a number.
#pragma once

#include "paged.h"

namespace jup {

typedef unsigned char u8;

// CODE: JUP_I8 or JUP_E4M3
template <int CODE>
constexpr float kTopCode = CODE == JUP_I8 ? 127.0f : 448.0f;
constexpr float kLeastMaximum = 0x1p-100f;  // of a head's values: T / m and m / T are then ordinary numbers, and zeros need no care

// Four numbers to the nearest codes (ties to even), the first in the lowest byte.  |x| <= T but for a rounding of x * (T / m), which rounds back.
template <int CODE>
__device__ __forceinline__ unsigned codes_of(const float* x) {
    if constexpr (CODE == JUP_I8) {
        unsigned w = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) w |= ((unsigned)(int)rintf(x[e]) & 0xFFu) << (8 * e);
        return w;
    } else {
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
        return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], lo, true);
    }
}

// The numbers of four codes.
template <int CODE>
__device__ __forceinline__ void numbers_of(unsigned w, float* x) {
    if constexpr (CODE == JUP_I8) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (float)(signed char)(w >> (8 * e));
    } else {
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        x[0] = lo[0]; x[1] = lo[1]; x[2] = hi[0]; x[3] = hi[1];
    }
}

// The same as bf16, which holds every code exactly.
template <int CODE>
__device__ __forceinline__ u32x2 bf16_of(unsigned w) {
    if constexpr (CODE == JUP_I8) {
        float x[4];
        numbers_of<CODE>(w, x);
        return (u32x2){pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
    } else {
        return (u32x2){__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false)),
                       __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true))};
    }
}

// x * y, 0 where x or y is (the instruction by its intrinsic, which has no builtin: the compiler knows what waits it needs).
__device__ float product_or_0(float x, float y) __asm("llvm.amdgcn.fmul.legacy");
// A probability times the scale of its value: 0 where the probability is, whatever the scale holds (a key that the row does not see).
__device__ __forceinline__ float scaled(float p, float scale) { return product_or_0(p, scale); }

}  // namespace jup
