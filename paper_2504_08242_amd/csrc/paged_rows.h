// Rotation of a step's rows on their way into their slots (paged_tables.hip, paged_codes.hip).
#pragma once

#include "paged.h"

namespace jup {

// The rotation turns the pair (x_i, x_(i + D/2)) by position * theta^(-2i/D).  The host hands over the turns per position,
// theta^(-2i/D) / 2 pi in 64 bits (one pow() and products), and a thread takes the fraction of a turn that is left in 64
// bits too: at position 10^6 the angle has lost 10^-10 of a turn.  Sine and cosine are fp32, as is the rotation; one rounding
// at the end.
struct Turns {
    double per_position[128];
};
__device__ __forceinline__ float2 turn(int position, double per_position) {
    const double t = (double)position * per_position;
    float s, c;
    sincospif(2.0f * (float)(t - rint(t)), &s, &c);
    return make_float2(c, s);
}

// (rope_theta 0: nothing is rotated)
inline Turns turns_of(float rope_theta, int head_dim) {
    Turns turns;
    const int half = head_dim / 2;
    if (rope_theta > 0.0f) {
        const double step = pow((double)rope_theta, -1.0 / half);
        double t = 0.15915494309189533577;  // 1 / 2 pi
        for (int i = 0; i < half; ++i, t *= step) turns.per_position[i] = t;
    }
    return turns;
}

// x, y: the eight values of lo and hi, rotated against each other
__device__ __forceinline__ void rotate8(const u32x4 lo, const u32x4 hi, const float2* cs, float* x, float* y) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float a = bf2f((u16)(lo[e / 2] >> (16 * (e & 1)))), b = bf2f((u16)(hi[e / 2] >> (16 * (e & 1))));
        x[e] = a * cs[e].x - b * cs[e].y;
        y[e] = b * cs[e].x + a * cs[e].y;
    }
}
__device__ __forceinline__ void rotate8(const u32x4 lo, const u32x4 hi, const float2* cs, u32x4& out_lo, u32x4& out_hi) {
    float x[8], y[8];
    rotate8(lo, hi, cs, x, y);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        out_lo[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
        out_hi[e] = pack_bf16x2(y[2 * e], y[2 * e + 1]);
    }
}

}  // namespace jup
