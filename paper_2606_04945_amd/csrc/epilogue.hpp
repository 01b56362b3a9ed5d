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
#include "tile_common.hpp"

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

// act(t).  silu(t) = t / (1 + exp2(-t log2 e));  gelu_tanh(t) = t (1 + tanh u) / 2 = t / (1 + e^(-2u)),
// u = sqrt(2 / pi) (t + 0.044715 t^3).
template <int ACT>
__device__ __forceinline__ float activated(float t) {
    if constexpr (ACT == kActSilu) return over_exp2(t, t * -1.44269504f);
    if constexpr (ACT == kActGeluTanh) return over_exp2(t, t * __builtin_fmaf(t * t, -0.102943240f, -2.30220820f));
    if constexpr (ACT == kActGelu) return gelu_erf(t);
    if constexpr (ACT == kActRelu || ACT == kActRelu2) {
        const float r = t < 0.0f ? 0.0f : t;             // a NaN stays one
        return ACT == kActRelu2 ? r * r : r;
    }
    return t;
}

template <int ACT>
struct ActIs {
    static constexpr int value = ACT;
};
// f with the activation as a constant, so that one branch serves a whole epilogue.
template <class F>
__device__ __forceinline__ void with_act(int act, F f) {
    switch (act) {
        case kActRelu: f(ActIs<kActRelu>()); break;
        case kActRelu2: f(ActIs<kActRelu2>()); break;
        case kActSilu: f(ActIs<kActSilu>()); break;
        case kActGelu: f(ActIs<kActGelu>()); break;
        case kActGeluTanh: f(ActIs<kActGeluTanh>()); break;
        default: f(ActIs<kActNone>()); break;
    }
}

// Rows of the residual, or of Y, as buffers: what lies past the last row or output is read as zeros
// and not written, and so is a residual that is not there, so nothing branches and the loads
// of an epilogue are in flight together (with a branch for each the compiler waits for one before it
// asks for the next: 16 x 4096 x 4096 with a residual 5.5 us against 4.7).  Offsets are of entries,
// in 32 bits: a caller's rows times their length are at most 2^29 (the host limits N).
struct RowsBuffer {
    __amdgpu_buffer_rsrc_t r;
    int shift;                                           // log2 of an entry's bytes
    // from row `row0` on, `rows` of them (none if negative) of `length` entries
    __device__ __forceinline__ RowsBuffer(const void* p, int f32, int row0, int rows, int length) {
        shift = f32 ? 2 : 1;
        const uint8_t* base = static_cast<const uint8_t*>(p);
        if (p) base += ((size_t)row0 * length) << shift;
        r = make_rsrc(base, p && rows > 0 ? (uint32_t)(rows * length) << shift : 0u);
    }
};
// Adding this leaves every value as it is, a zero's sign too.
__device__ __forceinline__ float neutral_if(bool none, float v) {
    return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, v) | (none ? 0x80000000u : 0u));
}

// Four consecutive entries of the residual, as read.
struct Res4 {
    uint2 lo, hi;                                        // fp16: lo; fp32: both
};
__device__ __forceinline__ uint2 load_b64(const __amdgpu_buffer_rsrc_t& r, uint32_t at) {
    return __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(r, (int)at, 0, 0));
}
__device__ __forceinline__ Res4 res_load(const RowsBuffer& b, uint32_t entry, bool in) {
    const uint32_t at = in ? entry << b.shift : kOOB;
    return Res4{load_b64(b.r, at), load_b64(b.r, b.shift == 2 ? at + 8 : kOOB)};
}
__device__ __forceinline__ void res_add(const EpilogueArgs& a, const Res4& r, float (&y)[4]) {
    const bool f32 = a.f32, none = a.res == nullptr;
    const float v0 = f32 ? __builtin_bit_cast(float, r.lo.x) : lo_h(r.lo.x);
    const float v1 = f32 ? __builtin_bit_cast(float, r.lo.y) : hi_h(r.lo.x);
    const float v2 = f32 ? __builtin_bit_cast(float, r.hi.x) : lo_h(r.lo.y);
    const float v3 = f32 ? __builtin_bit_cast(float, r.hi.y) : hi_h(r.lo.y);
    y[0] += neutral_if(none, v0), y[1] += neutral_if(none, v1);
    y[2] += neutral_if(none, v2), y[3] += neutral_if(none, v3);
}
__device__ __forceinline__ void out_store4(const RowsBuffer& b, uint32_t entry, bool in, const float (&y)[4]) {
    const uint32_t at = in ? entry << b.shift : kOOB;
    if (b.shift == 2) {
        v4i w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = __builtin_bit_cast(int, y[e]);
        __builtin_amdgcn_raw_buffer_store_b128(w, b.r, (int)at, 0, 0);
    } else {
        const uint32_t y0 = f2h(y[0]), y1 = f2h(y[1]), y2 = f2h(y[2]), y3 = f2h(y[3]);
        typedef uint32_t u2 __attribute__((ext_vector_type(2)));
        __builtin_amdgcn_raw_buffer_store_b64(u2{y0 | (y1 << 16), y2 | (y3 << 16)}, b.r, (int)at, 0, 0);
    }
}

// One entry: as a word that holds it (rows are of an even number of entries), then as a value.
__device__ __forceinline__ uint32_t res_load_one(const RowsBuffer& b, uint32_t entry, bool in) {
    return (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(b.r, (int)(in ? (entry << b.shift) & ~3u : kOOB), 0, 0);
}
__device__ __forceinline__ float res_one(const EpilogueArgs& a, uint32_t word, uint32_t entry) {
    const float h = entry & 1 ? hi_h(word) : lo_h(word);
    return neutral_if(a.res == nullptr, a.f32 ? __builtin_bit_cast(float, word) : h);
}
__device__ __forceinline__ void out_store_one(const RowsBuffer& b, uint32_t entry, bool in, float y) {
    const uint32_t at = in ? entry << b.shift : kOOB;
    if (b.shift == 2)
        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, y), b.r, (int)at, 0, 0);
    else
        __builtin_amdgcn_raw_buffer_store_b16(f2h(y), b.r, (int)at, 0, 0);
}

// Four entries of the bias from a buffer of it (an empty one where there is none).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t bias_buffer(const EpilogueArgs& a, int N) {
    return make_rsrc(a.bias, a.bias ? (uint32_t)N * 2 : 0u);
}
__device__ __forceinline__ void bias_add(const EpilogueArgs& a, const uint2& h, float (&t)[4]) {
    const bool none = a.bias == nullptr;
    t[0] += neutral_if(none, lo_h(h.x)), t[1] += neutral_if(none, hi_h(h.x));
    t[2] += neutral_if(none, lo_h(h.y)), t[3] += neutral_if(none, hi_h(h.y));
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
    const int other = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x128, 0xf, 0xf, false);
    return __builtin_bit_cast(float, other);
}

}  // namespace
}  // namespace sq
