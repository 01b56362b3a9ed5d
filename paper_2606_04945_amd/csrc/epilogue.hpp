// What a product does with its sums before they are stored: the dequantised value alone,
// or bias, activation (gated or not) and residual on top of it.
//
//   t = dequantised sum + bias;   y = act(t), or act(t_gate) t_up;   Y = round(y + residual)
//
// all in fp32, rounded once to Y's type.  Kernels take one of two types as their
// template parameter E:
//   Dequant       nothing more (an empty argument; Y is fp16, int32 sums optional);
//   Fused<GLU>    the above.  With GLU the weight rows alternate in blocks of 8 gates and
//                 their 8 ups within each group of 16 (weights_to_frag_kernel), while
//                 scales and bias keep the order [gates, ups]: a group's products of one
//                 row then lie in one wave, gate and up a fixed number of lanes apart.
#pragma once
#include "sq_internal.hpp"

namespace sq {

// Activations, by the header's numbers.
enum Act { kActNone = 0, kActRelu = 1, kActRelu2 = 2, kActSilu = 3, kActGelu = 4, kActGeluTanh = 5 };
constexpr int kActs = 6;

// Arguments of a fused epilogue as the host passes them.  `res` has Y's type; Y may be it.
struct EpilogueArgs {
    const uint16_t* bias;      // [N] fp16 in the order of the scales, or NULL
    const void* res;           // [M][out] fp16 or fp32, or NULL
    void* Y;                   // [M][out] fp16 or fp32
    int act;
    int f32;                   // type of res and Y
};

namespace {

struct Dequant {
    static constexpr bool kFused = false, kGlu = false;
};
template <bool GLU>
struct Fused {
    static constexpr bool kFused = true, kGlu = GLU;
    EpilogueArgs a;
};

// Where group `grp` of 16 weight rows has row `r`'s scale and bias (N rows in all).
template <bool GLU>
__device__ __forceinline__ int scale_index(int grp, int r, int N) {
    return GLU ? 8 * grp + (r & 7) + (r & 8 ? N / 2 : 0) : 16 * grp + r;
}

// t Phi(t).  Phi(-|t|) = erfc(z) / 2 with z = |t| / sqrt 2; erfc(z) = x exp2(P(x) - z^2 log2 e),
// x = 1 / (1 + 0.4 z), P of degree 8 fitted to log2(erfcx(z) / x) at Chebyshev points for z <= 10.5
// (largest error 1.1e-7; evaluated in fp32 Phi is within 7.5e-6 of its value down to t = -13, 1e-6 from -3 on).
__device__ __forceinline__ float gelu_erf(float t) {
    const float z = fabsf(t) * 0.70710678f;
    const float x = __builtin_amdgcn_rcpf(__builtin_fmaf(z, 0.4f, 1.0f));
    float p = -0.30781943f;
    p = __builtin_fmaf(p, x, 1.3754513f);
    p = __builtin_fmaf(p, x, -2.2300234f);
    p = __builtin_fmaf(p, x, 1.5403754f);
    p = __builtin_fmaf(p, x, -0.70806532f);
    p = __builtin_fmaf(p, x, 0.46233091f);
    p = __builtin_fmaf(p, x, 0.56940200f);
    p = __builtin_fmaf(p, x, 1.4461634f);
    p = __builtin_fmaf(p, x, -2.1478150f);
    const float q = 0.5f * x * __builtin_amdgcn_exp2f(__builtin_fmaf(t * t, -0.72134752f, p));
    return t * (t < 0.0f ? q : 1.0f - q);
}

// t / (1 + exp2(p)): past the range of exp2 the quotient is 0 or t.
__device__ __forceinline__ float over_exp2(float t, float p) {
    return t * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(p));
}

// act(t), four at a time: `act` is the same for all, so one branch serves them.
// silu(t) = t / (1 + exp2(-t log2 e));  gelu_tanh(t) = t (1 + tanh u) / 2 = t / (1 + e^(-2u)),
// u = sqrt(2 / pi) (t + 0.044715 t^3).
__device__ __forceinline__ void activate(float (&t)[4], int act) {
    if (act == kActSilu) {
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = over_exp2(t[e], t[e] * -1.44269504f);
    } else if (act == kActGeluTanh) {
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = over_exp2(t[e], t[e] * __builtin_fmaf(t[e] * t[e], -0.102943240f, -2.30220820f));
    } else if (act == kActGelu) {
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = gelu_erf(t[e]);
    } else if (act != kActNone) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float r = t[e] < 0.0f ? 0.0f : t[e];      // a NaN stays one
            t[e] = act == kActRelu2 ? r * r : r;
        }
    }
}

// Four consecutive entries of the residual, as read and as values.
struct Res4 {
    uint4 raw;
};
__device__ __forceinline__ Res4 res_load(const EpilogueArgs& a, size_t o) {
    Res4 r{make_uint4(0, 0, 0, 0)};
    if (a.f32) {
        r.raw = *reinterpret_cast<const uint4*>(static_cast<const float*>(a.res) + o);
    } else {
        const uint2 h = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(a.res) + o);
        r.raw.x = h.x, r.raw.y = h.y;
    }
    return r;
}
__device__ __forceinline__ void res_add(const EpilogueArgs& a, const Res4& r, float (&y)[4]) {
    if (a.f32) {
        y[0] += __builtin_bit_cast(float, r.raw.x), y[1] += __builtin_bit_cast(float, r.raw.y);
        y[2] += __builtin_bit_cast(float, r.raw.z), y[3] += __builtin_bit_cast(float, r.raw.w);
    } else {
        y[0] += h2f((uint16_t)(r.raw.x & 0xFFFFu)), y[1] += h2f((uint16_t)(r.raw.x >> 16));
        y[2] += h2f((uint16_t)(r.raw.y & 0xFFFFu)), y[3] += h2f((uint16_t)(r.raw.y >> 16));
    }
}
__device__ __forceinline__ void out_store4(const EpilogueArgs& a, size_t o, const float (&y)[4]) {
    if (a.f32) {
        *reinterpret_cast<float4*>(static_cast<float*>(a.Y) + o) = make_float4(y[0], y[1], y[2], y[3]);
    } else {
        const uint32_t y0 = f2h(y[0]), y1 = f2h(y[1]), y2 = f2h(y[2]), y3 = f2h(y[3]);
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.Y) + o) = make_uint2(y0 | (y1 << 16), y2 | (y3 << 16));
    }
}

// One entry.
__device__ __forceinline__ float res_one(const EpilogueArgs& a, size_t o) {
    return a.f32 ? static_cast<const float*>(a.res)[o] : h2f(static_cast<const uint16_t*>(a.res)[o]);
}
__device__ __forceinline__ void out_store_one(const EpilogueArgs& a, size_t o, float y) {
    if (a.f32)
        static_cast<float*>(a.Y)[o] = y;
    else
        static_cast<uint16_t*>(a.Y)[o] = f2h(y);
}

__device__ __forceinline__ float4 bias4(const uint16_t* b) {
    const uint2 h = *reinterpret_cast<const uint2*>(b);
    return make_float4(h2f((uint16_t)(h.x & 0xFFFFu)), h2f((uint16_t)(h.x >> 16)), h2f((uint16_t)(h.y & 0xFFFFu)),
                       h2f((uint16_t)(h.y >> 16)));
}

// The partner's value 32 lanes away: on return a and b hold, in lanes 0 .. 31, what a held there and what a
// held in lanes 32 .. 63; in lanes 32 .. 63 the same of b.
__device__ __forceinline__ void pair_halves(float& a, float& b) {
    const auto s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
                                                    false, false);
    const uint32_t s0 = s[0], s1 = s[1];
    a = __builtin_bit_cast(float, s0), b = __builtin_bit_cast(float, s1);
}

// The value 8 lanes away in a row of 16.
__device__ __forceinline__ float row_other_half(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x128, 0xf, 0xf, false));
}

}  // namespace
}  // namespace sq
