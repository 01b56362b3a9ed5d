// Norm with the residual stream around it, and the quantiser behind it:
//   u  = y,  or  (y - mean) r(y) w_post;   u = u gate;   h' = round(h + u alpha)
//   n  = (h' - mean) r(h') w;   n = n (1 + scale) + shift
//   X  = fp16(n),  or the codes of the gated n (as sgat_quantize on fp32 rows)
// with r(x) = 1 / sqrt(mean((x - mean)^2) + eps), the means taken off where asked.
//
// Sums are in fp64 (an entry costs one conversion and one fused multiply-add at the fp32
// rate, which the memory traffic hides) and the mean and r are rounded once to fp32, so
// neither depends on the order of the sum but where a rounding border lies within
// 2^-50 of it; every further step is one fp32 operation.  So the codes, which move where a
// value crosses a border, do not depend on how a row is shared out.
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
    v = __builtin_bit_cast(double, ((uint64_t)hi[0] << 32) | lo[0]) + __builtin_bit_cast(double, ((uint64_t)hi[1] << 32) | lo[1]);
    b = __builtin_bit_cast(uint64_t, v);
    lo = __builtin_amdgcn_permlane32_swap((uint32_t)b, (uint32_t)b, false, false);
    hi = __builtin_amdgcn_permlane32_swap((uint32_t)(b >> 32), (uint32_t)(b >> 32), false, false);
    return __builtin_bit_cast(double, ((uint64_t)hi[0] << 32) | lo[0]) + __builtin_bit_cast(double, ((uint64_t)hi[1] << 32) | lo[1]);
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

// Sums and maxima over the waves that share a row, each through a place of its own in LDS.
constexpr int kMaxWaves = 16, kExchanges = 5;
template <bool SHARED>
struct Row {
    double (*red)[kMaxWaves];
    int wave, waves, lane, used;
    __device__ __forceinline__ double sum(double v) {
        v = wave_sum(v);
        if constexpr (!SHARED) return v;
        if (lane == 0) red[used][wave] = v;
        __syncthreads();
        double s = red[used][0];
        for (int w = 1; w < waves; ++w) s += red[used][w];
        ++used;
        return s;
    }
    __device__ __forceinline__ float most(float v) {
        v = wave_most(v);
        if constexpr (!SHARED) return v;
        if (lane == 0) red[used][wave] = v;
        __syncthreads();
        float s = (float)red[used][0];
        for (int w = 1; w < waves; ++w) s = __builtin_elementwise_maximum(s, (float)red[used][w]);
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

// A lane's vectors of 8 entries: number i is vector lane + i lanes of the row; past the row
// loads give zeros, so every lane runs the same code.
template <int NV, bool F32, bool SHARED>
__global__ __launch_bounds__(SHARED ? 1024 : 64 * kRowsPerGroup) void norm_kernel(NormArgs a, int M, int K) {
    __shared__ double red[kExchanges][kMaxWaves];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int row = SHARED ? (int)blockIdx.x : (int)blockIdx.x * kRowsPerGroup + wave;
    if (!SHARED && row >= M) return;
    const int lanes = SHARED ? blockDim.x : kWave, t = SHARED ? threadIdx.x : lane;
    Row<SHARED> group{red, wave, (int)blockDim.x / kWave, lane, 0};

    const int64_t at = (int64_t)row * K;
    const uint32_t bytes = (uint32_t)K * 2;
    int seq = 0;
    if (a.seq) seq = min(max(a.seq[row], 0), a.seqs - 1);
    auto rows = [&](const uint16_t* p, int64_t offset) { return make_rsrc(p ? p + offset : p, p ? bytes : 0u); };
    const __amdgpu_buffer_rsrc_t rH = F32 ? make_rsrc(static_cast<const float*>(a.h) + at, 2 * bytes)
                                          : make_rsrc(static_cast<const uint16_t*>(a.h) + at, bytes);
    const __amdgpu_buffer_rsrc_t rY = rows(a.y, at), rP = rows(a.post, 0), rG = rows(a.gate, seq * a.gate_row);
    const __amdgpu_buffer_rsrc_t rW = rows(a.weight, 0), rS = rows(a.scale, seq * a.scale_row);
    const __amdgpu_buffer_rsrc_t rB = rows(a.shift, seq * a.shift_row);
    auto load = [&](const __amdgpu_buffer_rsrc_t& r, int i) {
        return __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(r, (t + i * lanes) * 16, 0, 0));
    };

    v4i yr[NV], hr[NV][F32 ? 2 : 1];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if constexpr (F32) {
            hr[i][0] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(rH, (t + i * lanes) * 32, 0, 0));
            hr[i][1] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(rH, (t + i * lanes) * 32 + 16, 0, 0));
        } else {
            hr[i][0] = load(rH, i);
        }
    }
    if (a.y) {
#pragma unroll
        for (int i = 0; i < NV; ++i) yr[i] = load(rY, i);
    }

    // mean (or 0) and r of rows x, whose entries past K are zeros
    auto statistics = [&](const float (&x)[NV][8], float& mean, float& rate) {
        double centre = 0.0, squares = 0.0;
        if (a.center) {
            double s = 0.0;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int q = 0; q < 8; ++q) s += (double)x[i][q];
            centre = group.sum(s) / K;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const bool in = (t + i * lanes) * 8 < K;
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const double d = in ? (double)x[i][q] - centre : 0.0;
                    squares = __builtin_fma(d, d, squares);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int q = 0; q < 8; ++q) squares = __builtin_fma((double)x[i][q], (double)x[i][q], squares);
        }
        squares = group.sum(squares);
        mean = (float)centre;
        rate = (float)(1.0 / __builtin_sqrt(squares / K + a.eps));
    };

    float x[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if constexpr (F32) {
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const int b = hr[i][q / 4][q % 4];
                x[i][q] = __builtin_bit_cast(float, b);
            }
        } else {
            halves(hr[i][0], x[i]);
        }
    }
    if (a.y) {
        float u[NV][8];
#pragma unroll
        for (int i = 0; i < NV; ++i) halves(yr[i], u[i]);
        if (a.post) {
            float mean, rate;
            statistics(u, mean, rate);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float w[8];
                halves(load(rP, i), w);
#pragma unroll
                for (int q = 0; q < 8; ++q) u[i][q] = (a.center ? u[i][q] - mean : u[i][q]) * rate * w[q];
            }
        }
        if (a.gate) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float w[8];
                halves(load(rG, i), w);
#pragma unroll
                for (int q = 0; q < 8; ++q) u[i][q] *= w[q];
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                x[i][q] += u[i][q] * a.alpha;
                if (!F32) x[i][q] = h2f(f2h(x[i][q]));
            }
    }
    if (a.h_out) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = t + i * lanes;
            if (v * 8 >= K) continue;
            if constexpr (F32) {
                float4* p = reinterpret_cast<float4*>(static_cast<float*>(a.h_out) + at + v * 8);
                p[0] = make_float4(x[i][0], x[i][1], x[i][2], x[i][3]);
                p[1] = make_float4(x[i][4], x[i][5], x[i][6], x[i][7]);
            } else {
                v4i w;
#pragma unroll
                for (int q = 0; q < 4; ++q) w[q] = (int)((uint32_t)f2h(x[i][2 * q]) | ((uint32_t)f2h(x[i][2 * q + 1]) << 16));
                *reinterpret_cast<v4i*>(static_cast<uint16_t*>(a.h_out) + at + v * 8) = w;
            }
        }
    }
    if (!a.X && !a.codes) return;

    float mean, rate;
    statistics(x, mean, rate);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int q = 0; q < 8; ++q) x[i][q] = (a.center ? x[i][q] - mean : x[i][q]) * rate;
        if (a.weight) {
            float w[8];
            halves(load(rW, i), w);
#pragma unroll
            for (int q = 0; q < 8; ++q) x[i][q] *= w[q];
        }
        if (a.scale) {
            float w[8];
            halves(load(rS, i), w);
#pragma unroll
            for (int q = 0; q < 8; ++q) x[i][q] *= 1.0f + w[q];
        }
        if (a.shift) {
            float w[8];
            halves(load(rB, i), w);
#pragma unroll
            for (int q = 0; q < 8; ++q) x[i][q] += w[q];
        }
    }
    if (a.X) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = t + i * lanes;
            if (v * 8 >= K) continue;
            v4i w;
#pragma unroll
            for (int q = 0; q < 4; ++q) w[q] = (int)((uint32_t)f2h(x[i][2 * q]) | ((uint32_t)f2h(x[i][2 * q + 1]) << 16));
            *reinterpret_cast<v4i*>(a.X + at + v * 8) = w;
        }
    }
    if (!a.codes) return;

    // the gate keeps columns [0, lim0) and [lim1, K)
    const bool masked = a.state ? a.state[row] != 0 : false;
    const int lim0 = a.state ? (masked ? K - a.d_u : K - a.d_m - a.d_u) : K, lim1 = masked ? K : K - a.d_u;
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (t + i * lanes) * 8;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            x[i][q] = (c + q < K) & ((c + q < lim0) | (c + q >= lim1)) ? x[i][q] : 0.0f;
            most = __builtin_elementwise_maximum(most, fabsf(x[i][q]));
        }
    }
    most = group.most(most);
    // a row with an entry that is not finite: scale NaN, zero codes
    const bool finite = most < __builtin_inff();
    const float s = finite ? most / (a.bits == 4 ? 7.0f : 127.0f) : __builtin_nanf("");
    const float inv = s > 0.0f ? 1.0f / s : 0.0f;
    if (t == 0) a.s[row] = s;
    uint8_t* cr = a.codes + (a.bits == 4 ? at / 2 : at);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = t + i * lanes;
        if (v * 8 >= K) continue;
        uint32_t lo = 0, hi = 0;
        if (a.bits == 4) {
            if (s > 0.0f) {
                int c[8];
                quant_codes8<7>(x[i], s, inv, c);
#pragma unroll
                for (int q = 0; q < 8; ++q) lo |= (uint32_t)(c[q] & 15) << (4 * q);
            }
            reinterpret_cast<uint32_t*>(cr)[v] = lo;
        } else {
            if (s > 0.0f) {
                int c[8];
                quant_codes8<127>(x[i], s, inv, c);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    lo |= (uint32_t)(c[q] & 255) << (8 * q);
                    hi |= (uint32_t)(c[4 + q] & 255) << (8 * q);
                }
            }
            reinterpret_cast<uint2*>(cr)[v] = make_uint2(lo, hi);
        }
    }
}

template <int NV, bool F32>
hipError_t launch(const NormArgs& a, int M, int K, int waves, hipStream_t st) {
    if (waves == 1)
        hipLaunchKernelGGL((norm_kernel<NV, F32, false>), dim3((M + kRowsPerGroup - 1) / kRowsPerGroup),
                           dim3(kWave * kRowsPerGroup), 0, st, a, M, K);
    else
        hipLaunchKernelGGL((norm_kernel<NV, F32, true>), dim3(M), dim3(kWave * waves), 0, st, a, M, K);
    return hipGetLastError();
}

template <bool F32>
hipError_t launch_nv(const NormArgs& a, int M, int K, hipStream_t st) {
    const NormPlan p = norm_plan(M, K);
    switch (p.nv) {
        case 1: return launch<1, F32>(a, M, K, p.waves, st);
        case 2: return launch<2, F32>(a, M, K, p.waves, st);
        case 4: return launch<4, F32>(a, M, K, p.waves, st);
        default: return hipErrorInvalidConfiguration;
    }
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, int M, int K, hipStream_t st) {
    return a.f32 ? launch_nv<true>(a, M, K, st) : launch_nv<false>(a, M, K, st);
}

}  // namespace sq
