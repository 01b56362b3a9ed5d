// Weight-only products: few fp16 rows times 4-bit weights with one fp16 scale per
// group of `group` inputs,
//   Y[m][n] = fp16(sum_G s[G][n] sum_{k in G} X[m][k] q[n][k]),
// and the quantiser of such weights.
//
// With few rows the call reads N K / 2 bytes of codes and little else, so the
// weights come in fragment order (1 KB contiguous for 16 rows x 128 codes) and each
// byte is read once.  Codes become halves in registers (exact), the fp16 matrix
// cores sum a group's products in fp32, and the group's scale is applied to that
// fp32 sum.
#include "tile_common.hpp"

namespace sq {
namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));

// The 8 codes of a word as halves in the order 0 4 1 5 2 6 3 7.  A flipped sign bit
// makes nibble u = code + 8; the half 0x6400 | u is 1024 + u, and 0x6400 | 16 u,
// taken where the nibble sits four bits up, is 1024 + 16 u, a sixteenth of which is
// 64 + u.
__device__ __forceinline__ h8 nibbles_to_halves(uint32_t w) {
    const uint32_t u = w ^ 0x88888888u, v = u >> 8;
    const h2 low = {(_Float16)1032.0f, (_Float16)1032.0f};
    const h2 sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f}, high = {(_Float16)-72.0f, (_Float16)-72.0f};
    const h2 a = __builtin_bit_cast(h2, (u & 0x000F000Fu) | 0x64006400u) - low;
    const h2 b = __builtin_elementwise_fma(__builtin_bit_cast(h2, (u & 0x00F000F0u) | 0x64006400u), sixteenth, high);
    const h2 c = __builtin_bit_cast(h2, (v & 0x000F000Fu) | 0x64006400u) - low;
    const h2 d = __builtin_elementwise_fma(__builtin_bit_cast(h2, (v & 0x00F000F0u) | 0x64006400u), sixteenth, high);
    return h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// 8 halves in the same order
__device__ __forceinline__ h8 same_order(v4i x) {
    v4i r;
    r[0] = (int)__builtin_amdgcn_perm((uint32_t)x[2], (uint32_t)x[0], 0x05040100u);
    r[1] = (int)__builtin_amdgcn_perm((uint32_t)x[2], (uint32_t)x[0], 0x07060302u);
    r[2] = (int)__builtin_amdgcn_perm((uint32_t)x[3], (uint32_t)x[1], 0x05040100u);
    r[3] = (int)__builtin_amdgcn_perm((uint32_t)x[3], (uint32_t)x[1], 0x07060302u);
    return __builtin_bit_cast(h8, r);
}

// One workgroup: NG groups of 16 outputs and up to 16 TM rows of X, the k steps of
// 128 dealt round to its waves, whose sums are added in LDS in the waves' order.
// GROUP: 32, 64 or 128 (a multiple of 128 applies one scale to several steps).
// In a fragment lane 16 j + r has the 32 codes of input group j of weight row r; a
// matrix instruction takes all its inputs from one such group instead, so that it
// never mixes scales: four lane-row exchanges per 32 codes.
template <int TM, int NG, int GROUP>
__global__ __launch_bounds__(512) void w4a16_kernel(const uint16_t* __restrict__ X, const uint8_t* __restrict__ Wf,
                                                    const uint16_t* __restrict__ s_w, int M, int N, int K, int group,
                                                    uint16_t* __restrict__ Y) {
    extern __shared__ __attribute__((aligned(16))) uint8_t sm[];
    constexpr int CH = 128 / GROUP, PER = 4 / CH;      // scales a step, matrix instructions a scale
    const int waves = blockDim.x / kWave;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r = lane % 16, g = lane / 16;
    const int groups = (N + 15) / 16, steps = (K + 127) / 128;
    const int g0 = blockIdx.x * NG, m0 = blockIdx.y * (16 * TM);
    const uint16_t* xr[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) xr[i] = X + (int64_t)min(m0 + 16 * i + r, M - 1) * K + 8 * g;
    f4 sum[NG][TM];
#pragma unroll
    for (int n = 0; n < NG; ++n)
#pragma unroll
        for (int i = 0; i < TM; ++i) sum[n][i] = f4{0, 0, 0, 0};
    for (int t = wave; t < steps; t += waves) {
        v4i w[NG];
        h8 x[TM][4];
        f4 sc[NG][CH];
#pragma unroll
        for (int n = 0; n < NG; ++n) {
            const int grp = min(g0 + n, groups - 1);
            w[n] = *reinterpret_cast<const v4i*>(Wf + ((int64_t)t * groups + grp) * 1024 + lane * 16);
#pragma unroll
            for (int z = 0; z < CH; ++z) {
                const int sg = min(t * 128 + z * GROUP, K - 1) / group;
                const uint2 s = *reinterpret_cast<const uint2*>(s_w + (int64_t)sg * N + min(grp * 16 + 4 * g, N - 4));
                sc[n][z] = f4{lo_h(s.x), hi_h(s.x), lo_h(s.y), hi_h(s.y)};
            }
        }
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int k = t * 128 + 32 * s;        // K is a multiple of 64: all of a chunk of 32 or none
                x[i][s] = k < K ? same_order(*reinterpret_cast<const v4i*>(xr[i] + k)) : h8{};
            }
#pragma unroll
        for (int n = 0; n < NG; ++n) {
            uint32_t c[4] = {(uint32_t)w[n][0], (uint32_t)w[n][1], (uint32_t)w[n][2], (uint32_t)w[n][3]};
            transpose_rows4(c[0], c[1], c[2], c[3]);
            h8 q[4];
#pragma unroll
            for (int s = 0; s < 4; ++s) q[s] = nibbles_to_halves(c[s]);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int z = 0; z < CH; ++z) {
                    f4 acc{0, 0, 0, 0};
#pragma unroll
                    for (int s = z * PER; s < (z + 1) * PER; ++s)
                        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(q[s], x[i][s], acc, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[n][i][e] = __builtin_fmaf(acc[e], sc[n][z][e], sum[n][i][e]);
                }
        }
    }
    f4* red = reinterpret_cast<f4*>(sm);               // [wave - 1][NG][TM][lane]
    if (wave > 0) {
#pragma unroll
        for (int n = 0; n < NG; ++n)
#pragma unroll
            for (int i = 0; i < TM; ++i) red[(((wave - 1) * NG + n) * TM + i) * kWave + lane] = sum[n][i];
    }
    __syncthreads();
    // the waves share the adding up: tile z of NG TM to wave z % waves
    if (wave == 0) {
#pragma unroll
        for (int n = 0; n < NG; ++n)
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                for (int v = 0; v < waves - 1; ++v) sum[n][i] += red[((v * NG + n) * TM + i) * kWave + lane];
                const int m = m0 + 16 * i + r, o = (g0 + n) * 16 + 4 * g;
                if (m < M && o < N) {
                    uint2 y;
                    y.x = (uint32_t)f2h(sum[n][i][0]) | ((uint32_t)f2h(sum[n][i][1]) << 16);
                    y.y = (uint32_t)f2h(sum[n][i][2]) | ((uint32_t)f2h(sum[n][i][3]) << 16);
                    *reinterpret_cast<uint2*>(Y + (int64_t)m * N + o) = y;
                }
            }
    }
}

// One wave: one group of one output channel.  The scale is rounded to fp16 first
// and the codes are taken against the rounded scale, so that code times scale is the
// nearest such value to the weight.
__global__ __launch_bounds__(256) void quantize_group_kernel(const uint16_t* __restrict__ W, int N, int K, int group,
                                                             uint8_t* __restrict__ Wq, uint16_t* __restrict__ s_w) {
    const int lane = threadIdx.x % kWave;
    const int64_t item = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
    const int ng = K / group;
    if (item >= (int64_t)N * ng) return;
    const int n = (int)(item / ng), gi = (int)(item % ng);
    const uint32_t* w = reinterpret_cast<const uint32_t*>(W + (int64_t)n * K + gi * group);
    float m = 0.0f;
    for (int e = lane; e < group / 2; e += kWave) m = fmaxf(m, fmaxf(fabsf(lo_h(w[e])), fabsf(hi_h(w[e]))));
    m = wave_max(m);
    const uint16_t sh = f2h(m / 7.0f);
    const float s = h2f(sh);
    uint8_t* q = Wq + ((int64_t)n * K + gi * group) / 2;
    for (int e = lane; e < group / 2; e += kWave) {
        const int a = s > 0.0f ? quant4(lo_h(w[e]), s) : 0, b = s > 0.0f ? quant4(hi_h(w[e]), s) : 0;
        q[e] = (uint8_t)((a & 15) | ((b & 15) << 4));
    }
    if (lane == 0) s_w[(int64_t)gi * N + n] = sh;
}

template <int TM, int NG>
hipError_t launch_tile(const uint16_t* X, const uint8_t* Wf, const uint16_t* s_w, int M, int N, int K, int group,
                       uint16_t* Y, int waves, hipStream_t st) {
    const dim3 grid((unsigned)(((N + 15) / 16 + NG - 1) / NG), (unsigned)((M + 16 * TM - 1) / (16 * TM)));
    const dim3 block(kWave * waves);
    const size_t lds = (size_t)(waves - 1) * NG * TM * kWave * sizeof(f4);
    if (group == 32)
        hipLaunchKernelGGL((w4a16_kernel<TM, NG, 32>), grid, block, lds, st, X, Wf, s_w, M, N, K, group, Y);
    else if (group == 64)
        hipLaunchKernelGGL((w4a16_kernel<TM, NG, 64>), grid, block, lds, st, X, Wf, s_w, M, N, K, group, Y);
    else
        hipLaunchKernelGGL((w4a16_kernel<TM, NG, 128>), grid, block, lds, st, X, Wf, s_w, M, N, K, group, Y);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_group(const uint16_t* W, int N, int K, int group, uint8_t* Wq, uint16_t* s_w,
                                 hipStream_t st) {
    const int64_t items = (int64_t)N * (K / group);
    hipLaunchKernelGGL(quantize_group_kernel, dim3((unsigned)((items + 3) / 4)), dim3(256), 0, st, W, N, K, group, Wq,
                       s_w);
    return hipGetLastError();
}

hipError_t launch_w4a16_frag(const uint16_t* X, const uint8_t* Wf, const uint16_t* s_w, int M, int N, int K, int group,
                             uint16_t* Y, hipStream_t st) {
    return launch_tile<1, 1>(X, Wf, s_w, M, N, K, group, Y, 8, st);
}

}  // namespace sq
