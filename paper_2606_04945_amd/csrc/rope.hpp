// Rotary positions: the rotation of one unit of a head's entries, shared by the
// kernels that rotate queries and keys.
//
// Pair j of a head turns by the angle pos f_j (f_j in radians per position):
// (u, v) -> a (u cos - v sin, v cos + u sin).  Pair j is entries (j, j + rot/2)
// in the half layout and (2j, 2j + 1) in the pairs layout; entries from rot on
// stay.  A far position's angle has more bits than an fp32 holds, so the turn is
// formed and reduced in fp64 and only what is left of it, at most half a turn,
// goes to fp32.
#pragma once
#include "serve.hpp"

namespace sq {

constexpr int kRopeHalf = 0, kRopePairs = 1;

namespace {

// cos and sin of pos f, times amp; transposed: the sine's sign flipped.
__device__ __forceinline__ void rope_angle(int pos, double f, float amp, bool transpose, float& c, float& s) {
    constexpr double kPerTurn = 0.15915494309189533577;   // 1 / (2 pi)
    const double t = (double)pos * (f * kPerTurn);
    const float h = 2.0f * (float)(t - __builtin_rint(t));   // half turns, in [-1, 1]
    float cc, ss;
    sincospif(h, &ss, &cc);
    c = cc * amp;
    s = transpose ? -(ss * amp) : ss * amp;
}

// A row of D entries as units of 2 VEC entries, each two runs of VEC: the first
// rot / (2 VEC) units hold VEC whole pairs each, the rest are not rotated.
struct RopeUnit {
    int a, b;      // first entries of the two runs
    int pair;      // first pair, or -1: not rotated
};

template <int VEC>
__device__ __forceinline__ RopeUnit rope_unit(int u, int rot, int layout) {
    const int turned = rot / (2 * VEC);
    if (u >= turned) {
        const int e = rot + (u - turned) * 2 * VEC;
        return {e, e + VEC, -1};
    }
    if (layout == kRopeHalf) return {u * VEC, rot / 2 + u * VEC, u * VEC};
    return {2 * u * VEC, 2 * u * VEC + VEC, u * VEC};
}

// Rotates one unit: a and b are its two runs, c and s the VEC angles.
template <int VEC>
__device__ __forceinline__ void rope_turn(float (&a)[VEC], float (&b)[VEC], const float (&c)[VEC],
                                          const float (&s)[VEC], int layout) {
    if (VEC == 1 || layout == kRopeHalf) {
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            const float u = a[q], v = b[q];
            a[q] = __builtin_fmaf(u, c[q], -(v * s[q]));
            b[q] = __builtin_fmaf(v, c[q], u * s[q]);
        }
    } else {
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            float& x = q < VEC / 2 ? a[(2 * q) % VEC] : b[(2 * q) % VEC];
            float& y = q < VEC / 2 ? a[(2 * q + 1) % VEC] : b[(2 * q + 1) % VEC];
            const float u = x, v = y;
            x = __builtin_fmaf(u, c[q], -(v * s[q]));
            y = __builtin_fmaf(v, c[q], u * s[q]);
        }
    }
}

template <int VEC>
__device__ __forceinline__ void load_run(const uint16_t* p, float (&x)[VEC]) {
    if constexpr (VEC == 8) {
        const v4i w = *reinterpret_cast<const v4i*>(p);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            x[2 * q] = h2f((uint16_t)((uint32_t)w[q] & 0xFFFFu));
            x[2 * q + 1] = h2f((uint16_t)((uint32_t)w[q] >> 16));
        }
    } else {
#pragma unroll
        for (int q = 0; q < VEC; ++q) x[q] = h2f(p[q]);
    }
}

template <int VEC>
__device__ __forceinline__ void store_run(uint16_t* p, const float (&x)[VEC]) {
    if constexpr (VEC == 8) {
        v4i w;
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = (int)((uint32_t)f2h(x[2 * q]) | ((uint32_t)f2h(x[2 * q + 1]) << 16));
        *reinterpret_cast<v4i*>(p) = w;
    } else {
#pragma unroll
        for (int q = 0; q < VEC; ++q) p[q] = f2h(x[q]);
    }
}

}  // namespace
}  // namespace sq
