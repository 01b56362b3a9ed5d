// Norm with the residual stream around it, and the quantiser behind it:
//   u  = y,  or  (y - mean) r(y) w_post;   u = u gate;   h' = round(h + u alpha)
//   n  = (h' - mean) r(h') w;   n = n (1 + scale) + shift
//   X  = fp16(n),  or the codes of the gated n (as sgat_quantize on fp32 rows)
// with r(x) = 1 / sqrt(mean((x - mean)^2) + eps), the means taken off where asked.
//
// Sums are in fp64 (an entry costs one conversion and one fused multiply-add at the fp32
// rate, which the memory traffic hides) and the mean and r are rounded once to fp32, so
// neither depends on the order of the sum but where a border of fp32's rounding lies within the sum's own
// error; every further step is one fp32 operation.  So the codes, which move where a
// value crosses a border, do not depend on how a row is shared out.  That error: an entry goes through at most
// 32 steps of a lane, 6 of a wave and 15 between waves, each 2^-53, so two orders differ by at most 106 2^-53 < 2^-46
// of a sum of squares; a mean by that much of the mean magnitude, r(x) by half of it where nothing is
// taken off.  With a mean taken off in one pass (see `statistics`) mean(x^2) is up to 17 times the variance and
// mean^2 errs twice, so r by 25 times that, 2^-42.
//
// A row is held in registers by one wave or by all waves of a workgroup: it is read once,
// every load of it in flight before the first sum.
#include "layer.hpp"
#include "norm_plan.hpp"
#include "tile_common.hpp"

namespace sq {
namespace {

constexpr int kRowsPerGroup = 4;       // rows of a workgroup whose waves have a row each

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false);
}
// The wave's sum (every lane has it): within quads, halves of rows, rows, then across rows.
template <int CTRL>
__device__ __forceinline__ double plus_dpp(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint64_t o = ((uint64_t)dpp<CTRL>((uint32_t)(b >> 32)) << 32) | dpp<CTRL>((uint32_t)b);
    return v + __builtin_bit_cast(double, o);
}
__device__ __forceinline__ double wave_sum(double v) {
    v = plus_dpp<0xB1>(v);             // lanes 1 0 3 2
    v = plus_dpp<0x4E>(v);             // lanes 2 3 0 1
    v = plus_dpp<0x141>(v);            // mirrored halves of a row
    v = plus_dpp<0x140>(v);            // mirrored rows
    uint64_t b = __builtin_bit_cast(uint64_t, v);
    auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)b, (uint32_t)b, false, false);
    auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(b >> 32), (uint32_t)(b >> 32), false, false);
    v = __builtin_bit_cast(double, ((uint64_t)hi[0] << 32) | lo[0]) +
        __builtin_bit_cast(double, ((uint64_t)hi[1] << 32) | lo[1]);
    b = __builtin_bit_cast(uint64_t, v);
    lo = __builtin_amdgcn_permlane32_swap((uint32_t)b, (uint32_t)b, false, false);
    hi = __builtin_amdgcn_permlane32_swap((uint32_t)(b >> 32), (uint32_t)(b >> 32), false, false);
    return __builtin_bit_cast(double, ((uint64_t)hi[0] << 32) | lo[0]) +
           __builtin_bit_cast(double, ((uint64_t)hi[1] << 32) | lo[1]);
}
// The wave's maximum of values that are not negative; a NaN wins.
template <int CTRL>
__device__ __forceinline__ float max_dpp(float v) {
    return __builtin_elementwise_maximum(v, __builtin_bit_cast(float, dpp<CTRL>(__builtin_bit_cast(uint32_t, v))));
}
__device__ __forceinline__ float wave_most(float v) {
    v = max_dpp<0xB1>(v);
    v = max_dpp<0x4E>(v);
    v = max_dpp<0x141>(v);
    v = max_dpp<0x140>(v);
    uint32_t b = __builtin_bit_cast(uint32_t, v);
    auto p = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    uint32_t p0 = p[0], p1 = p[1];
    v = __builtin_elementwise_maximum(__builtin_bit_cast(float, p0), __builtin_bit_cast(float, p1));
    b = __builtin_bit_cast(uint32_t, v);
    p = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    p0 = p[0], p1 = p[1];
    return __builtin_elementwise_maximum(__builtin_bit_cast(float, p0), __builtin_bit_cast(float, p1));
}

// Sums and maxima over the WAVES waves that share a row, each through a place of its own in LDS.
constexpr int kExchanges = 7;        // three for each of two norms, one for the largest entry
template <int WAVES>
struct Row {
    double (*red)[WAVES];
    int wave, lane, used;
    __device__ __forceinline__ double sum(double v) {
        v = wave_sum(v);
        if constexpr (WAVES == 1) return v;
        if (lane == 0) red[used][wave] = v;
        __syncthreads();
        double s = red[used][0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) s += red[used][w];
        ++used;
        return s;
    }
    __device__ __forceinline__ void sum(double& v, double& w) {
        v = wave_sum(v), w = wave_sum(w);
        if constexpr (WAVES == 1) return;
        if (lane == 0) red[used][wave] = v, red[used + 1][wave] = w;
        __syncthreads();
        v = red[used][0], w = red[used + 1][0];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) v += red[used][i], w += red[used + 1][i];
        used += 2;
    }
    __device__ __forceinline__ float most(float v) {
        v = wave_most(v);
        if constexpr (WAVES == 1) return v;
        if (lane == 0) red[used][wave] = v;
        __syncthreads();
        float s = (float)red[used][0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) s = __builtin_elementwise_maximum(s, (float)red[used][w]);
        ++used;
        return s;
    }
};

__device__ __forceinline__ void halves(const v4i& raw, float (&x)[8]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t w = (uint32_t)raw[q];
        x[2 * q] = lo_h(w), x[2 * q + 1] = hi_h(w);
    }
}
__device__ __forceinline__ v4i to_halves(const float (&x)[8]) {
    v4i w;
#pragma unroll
    for (int q = 0; q < 4; ++q) w[q] = (int)((uint32_t)f2h(x[2 * q]) | ((uint32_t)f2h(x[2 * q + 1]) << 16));
    return w;
}

// A vector of the stream in its own type: what a lane holds of it between the sums.
template <bool F32>
struct Held {
    v4i raw[F32 ? 2 : 1];
    __device__ __forceinline__ void get(float (&x)[8]) const {
        if constexpr (F32) {
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const int b = raw[q / 4][q % 4];       // copied out first: a bit cast of a vector element reads element 0
                x[q] = __builtin_bit_cast(float, b);
            }
        } else {
            halves(raw[0], x);
        }
    }
    __device__ __forceinline__ void put(const float (&x)[8]) {   // rounds to the stream's type
        if constexpr (F32) {
#pragma unroll
            for (int q = 0; q < 8; ++q) raw[q / 4][q % 4] = __builtin_bit_cast(int, x[q]);
        } else {
            raw[0] = to_halves(x);
        }
    }
};

// A lane's vectors of 8 entries: number i is vector lane + i lanes of the row; past the row
// loads give zeros, so every lane runs the same code.  FULL: norm of y, gate, scale, shift and
// means are possible; BITS: of the codes, 0 for none.
template <int NV, bool F32, int WAVES, bool FULL, int BITS>
__global__ __launch_bounds__(kWave * (WAVES == 1 ? kRowsPerGroup : WAVES)) void norm_kernel(NormArgs a, int M, int K) {
    constexpr bool SHARED = WAVES > 1;
    __shared__ double red[kExchanges][WAVES];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int row = SHARED ? (int)blockIdx.x : (int)blockIdx.x * kRowsPerGroup + wave;
    if (!SHARED && row >= M) return;
    constexpr int lanes = kWave * WAVES;
    const int t = SHARED ? threadIdx.x : lane;
    Row<WAVES> group{red, wave, lane, 0};
    const bool center = FULL && a.center;

    const int64_t at = (int64_t)row * K;
    const uint32_t bytes = (uint32_t)K * 2;
    struct Vectors {
        v4i raw[NV];
    };
    auto load = [&](const uint16_t* p, int i) {
        return __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(make_rsrc(p, bytes), (t + i * lanes) * 16, 0, 0));
    };
    auto request = [&](const uint16_t* p, int64_t offset, Vectors& f) {
        if (!p) return;
#pragma unroll
        for (int i = 0; i < NV; ++i) f.raw[i] = load(p + offset, i);
    };
    // Factors are requested ahead of the sum that their use waits for; where a lane holds four vectors of
    // each of six kinds they would not fit its registers, and are read as they are used.
    constexpr bool kAhead = !FULL || NV < 4;
    auto ahead = [&](const uint16_t* p, int64_t offset, Vectors& f) {
        if (kAhead) request(p, offset, f);
    };
    auto factors = [&](const uint16_t* p, int64_t offset, const Vectors& f, int i, float (&w)[8]) {
        halves(kAhead ? f.raw[i] : load(p + offset, i), w);
    };
    Held<F32> h[NV];
    Vectors y, post, gate, weight, scale, shift;
    const __amdgpu_buffer_rsrc_t rH = F32 ? make_rsrc(static_cast<const float*>(a.h) + at, 2 * bytes)
                                          : make_rsrc(static_cast<const uint16_t*>(a.h) + at, bytes);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int z = 0; z < (F32 ? 2 : 1); ++z)
            h[i].raw[z] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(
                              rH, (t + i * lanes) * (F32 ? 32 : 16) + 16 * z, 0, 0));
    request(a.y, at, y);
    int64_t seq = 0;
    if (FULL && a.seq) seq = min(max(a.seq[row], 0), a.seqs - 1);
    const bool masked = BITS != 0 && a.state && a.state[row] != 0;

    // Mean (or 0) and r of a row whose vector i is get(i, x); its entries past K are zeros.  With a
    // mean: both sums in one pass, mean(x^2) - mean^2 where that loses less than five bits (the difference is at
    // least a 17th of mean(x^2)), else the sum of (x - mean)^2 in another.
    auto statistics = [&](auto get, float& mean, float& rate) {
        double s = 0.0, squares = 0.0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float x[8];
            get(i, x);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const double d = (double)x[q];
                if (center) s += d;
                squares = __builtin_fma(d, d, squares);
            }
        }
        if (!center) {
            squares = group.sum(squares) / K;
        } else {
            group.sum(s, squares);
            s /= K;
            squares = squares / K - s * s;
            if (!(s * s <= 16.0 * squares)) {
                squares = 0.0;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const bool in = (t + i * lanes) * 8 < K;
                    float x[8];
                    get(i, x);
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        const double d = in ? (double)x[q] - s : 0.0;
                        squares = __builtin_fma(d, d, squares);
                    }
                }
                squares = group.sum(squares) / K;
            }
        }
        mean = (float)s;
        rate = (float)(1.0 / __builtin_sqrt(squares + a.eps));
    };

    if (a.y) {
        float mean = 0.0f, rate = 1.0f;
        if (FULL) {
            ahead(a.gate, seq * a.gate_row, gate);
            if (a.post) {
                ahead(a.post, 0, post);
                statistics([&](int i, float (&x)[8]) { halves(y.raw[i], x); }, mean, rate);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float x[8], u[8], w[8];
            halves(y.raw[i], u);
            if (FULL && a.post) {
                factors(a.post, 0, post, i, w);
#pragma unroll
                for (int q = 0; q < 8; ++q) u[q] = (center ? u[q] - mean : u[q]) * rate * w[q];
            }
            if (FULL && a.gate) {
                factors(a.gate, seq * a.gate_row, gate, i, w);
#pragma unroll
                for (int q = 0; q < 8; ++q) u[q] *= w[q];
            }
            h[i].get(x);
#pragma unroll
            for (int q = 0; q < 8; ++q) x[q] += u[q] * a.alpha;
            h[i].put(x);
        }
    }
    if (a.h_out) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = t + i * lanes;
            if (v * 8 >= K) continue;
            v4i* p = F32 ? reinterpret_cast<v4i*>(static_cast<float*>(a.h_out) + at + v * 8)
                         : reinterpret_cast<v4i*>(static_cast<uint16_t*>(a.h_out) + at + v * 8);
            p[0] = h[i].raw[0];
            if (F32) p[1] = h[i].raw[F32 ? 1 : 0];
        }
    }
    if (BITS == 0 && !a.X) return;

    ahead(a.weight, 0, weight);
    if (FULL) {
        ahead(a.scale, seq * a.scale_row, scale);
        ahead(a.shift, seq * a.shift_row, shift);
    }
    float mean, rate;
    statistics([&](int i, float (&x)[8]) { h[i].get(x); }, mean, rate);
    // the gate keeps columns [0, lim0) and [lim1, K)
    const int lim0 = a.state ? (masked ? K - a.d_u : K - a.d_m - a.d_u) : K, lim1 = masked ? K : K - a.d_u;
    float n[NV][8], most = 0.0f, lost = 0.0f;          // largest entry kept, and dropped
    auto drop = [&](const float (&x)[8]) {
#pragma unroll
        for (int q = 0; q < 8; ++q) lost = __builtin_elementwise_maximum(lost, fabsf(x[q]));
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = t + i * lanes;
        float(&x)[8] = n[i];
        float w[8];
        h[i].get(x);
#pragma unroll
        for (int q = 0; q < 8; ++q) x[q] = (center ? x[q] - mean : x[q]) * rate;
        if (a.weight) {
            factors(a.weight, 0, weight, i, w);
#pragma unroll
            for (int q = 0; q < 8; ++q) x[q] *= w[q];
        }
        if (FULL && a.scale) {
            factors(a.scale, seq * a.scale_row, scale, i, w);
#pragma unroll
            for (int q = 0; q < 8; ++q) x[q] *= 1.0f + w[q];
        }
        if (FULL && a.shift) {
            factors(a.shift, seq * a.shift_row, shift, i, w);
#pragma unroll
            for (int q = 0; q < 8; ++q) x[q] += w[q];
        }
        if (a.X && v * 8 < K) *reinterpret_cast<v4i*>(a.X + at + v * 8) = to_halves(x);
        if (BITS == 0) continue;
        // nearly every vector is kept or dropped whole (a masked row drops its u-band, an unmasked one its m-band);
        // past the row an entry is what the mean makes of a zero, and no part of it
        const int c = 8 * v;
        if ((c >= K) | ((c >= lim0) & (c + 8 <= lim1))) {
            if (c < K) drop(x);
#pragma unroll
            for (int q = 0; q < 8; ++q) x[q] = 0.0f;
        } else if ((c + 8 > lim0) & (c < lim1)) {
            drop(x);
#pragma unroll
            for (int q = 0; q < 8; ++q) x[q] = (c + q < lim0) | (c + q >= lim1) ? x[q] : 0.0f;
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) most = __builtin_elementwise_maximum(most, fabsf(x[q]));
    }
    if constexpr (BITS != 0) {
        constexpr int QMAX = BITS == 4 ? 7 : 127;
        // a row with an entry that is not finite, be it in a dropped band: scale NaN, zero codes (an infinity
        // there has made the rate and so every kept entry of an RMS norm 0)
        most = group.most(lost < __builtin_inff() ? most : __builtin_nanf(""));
        const float s = most < __builtin_inff() ? most / (float)QMAX : __builtin_nanf("");
        const float inv = s > 0.0f ? 1.0f / s : 0.0f;
        if (t == 0) a.s[row] = s;
        uint8_t* cr = a.codes + at * BITS / 8;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = t + i * lanes;
            if (v * 8 >= K) continue;
            uint32_t word[BITS / 4] = {};
            if (s > 0.0f) {
                int c[8];
                quant_codes8<QMAX>(n[i], s, inv, c);
#pragma unroll
                for (int q = 0; q < 8; ++q) word[q * BITS / 32] |= (uint32_t)(c[q] & (BITS == 4 ? 15 : 255)) << (BITS * q % 32);
            }
            if (BITS == 4)
                reinterpret_cast<uint32_t*>(cr)[v] = word[0];
            else
                reinterpret_cast<uint2*>(cr)[v] = make_uint2(word[0], word[BITS / 4 - 1]);
        }
    }
}

template <int NV, bool F32, int WAVES, bool FULL>
void launch(const NormArgs& a, int M, int K, hipStream_t st) {
    const dim3 grid(WAVES == 1 ? (M + kRowsPerGroup - 1) / kRowsPerGroup : M);
    const dim3 block(kWave * (WAVES == 1 ? kRowsPerGroup : WAVES));
    if (!a.codes)
        hipLaunchKernelGGL((norm_kernel<NV, F32, WAVES, FULL, 0>), grid, block, 0, st, a, M, K);
    else if (a.bits == 4)
        hipLaunchKernelGGL((norm_kernel<NV, F32, WAVES, FULL, 4>), grid, block, 0, st, a, M, K);
    else
        hipLaunchKernelGGL((norm_kernel<NV, F32, WAVES, FULL, 8>), grid, block, 0, st, a, M, K);
}

template <int NV, int WAVES>
hipError_t launch(const NormArgs& a, int M, int K, hipStream_t st) {
    const bool full = a.post || a.gate || a.scale || a.shift || a.center;
    if (a.f32 && full)
        launch<NV, true, WAVES, true>(a, M, K, st);
    else if (a.f32)
        launch<NV, true, WAVES, false>(a, M, K, st);
    else if (full)
        launch<NV, false, WAVES, true>(a, M, K, st);
    else
        launch<NV, false, WAVES, false>(a, M, K, st);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, int M, int K, hipStream_t st) {
    const NormPlan p = norm_plan(M, K);
    switch (p.waves * 8 + p.nv) {
        case 8 + 1: return launch<1, 1>(a, M, K, st);
        case 16 + 1: return launch<1, 2>(a, M, K, st);
        case 16 + 2: return launch<2, 2>(a, M, K, st);
        case 32 + 1: return launch<1, 4>(a, M, K, st);
        case 32 + 2: return launch<2, 4>(a, M, K, st);
        case 64 + 1: return launch<1, 8>(a, M, K, st);
        case 64 + 2: return launch<2, 8>(a, M, K, st);
        case 128 + 2: return launch<2, 16>(a, M, K, st);
        case 128 + 4: return launch<4, 16>(a, M, K, st);
        default: return hipErrorInvalidConfiguration;
    }
}

}  // namespace sq
