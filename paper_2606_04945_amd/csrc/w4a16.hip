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
#include "serve.hpp"
#include "tile_common.hpp"
#include "w4a16_plan.hpp"

namespace sq {
namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));

template <int I>
struct Index {
    static constexpr int value = I;
};

// The 8 codes of a word as halves in the order 0 4 1 5 2 6 3 7.  With its sign bit
// flipped a nibble is u = code + 8; the half 0x6400 | u is 1024 + u, and 0x6400 | 16 u,
// taken where the nibble sits four bits up, is 1024 + 16 u, a sixteenth of which is
// 64 + u.  Masking, flipping and the 0x64 are one three-operand instruction if the
// constants are registers.
struct NibbleMasks {
    uint32_t low, high, c_low, c_high;
};
__device__ __forceinline__ NibbleMasks nibble_masks() {
    NibbleMasks m{0x000F000Fu, 0x00F000F0u, 0x64086408u, 0x64806480u};
    asm volatile("" : "+v"(m.low), "+v"(m.high), "+v"(m.c_low), "+v"(m.c_high));
    return m;
}
__device__ __forceinline__ h8 nibbles_to_halves(uint32_t w, const NibbleMasks& k) {
    const uint32_t v = w >> 8;
    const h2 low = {(_Float16)1032.0f, (_Float16)1032.0f};
    const h2 sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f}, high = {(_Float16)-72.0f, (_Float16)-72.0f};
    const h2 a = __builtin_bit_cast(h2, (w & k.low) ^ k.c_low) - low;
    const h2 b = __builtin_elementwise_fma(__builtin_bit_cast(h2, (w & k.high) ^ k.c_high), sixteenth, high);
    const h2 c = __builtin_bit_cast(h2, (v & k.low) ^ k.c_low) - low;
    const h2 d = __builtin_elementwise_fma(__builtin_bit_cast(h2, (v & k.high) ^ k.c_high), sixteenth, high);
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

// lane n of each row of 16 lanes to the whole row
template <int LANE>
__device__ __forceinline__ uint32_t row_broadcast(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x150 + LANE, 0xf, 0xf, false);
}

// What a wave reads for one k step of 128: NG groups of 16 outputs, their scales (lane r
// of a row has group r % NG's), TM row tiles of X.
template <int TM, int NG, int CH>
struct Step {
    v4i w[NG], x[TM][4];
    uint2 s[CH];
};

// One workgroup: NG groups of 16 outputs and up to 16 TM rows of X, the k steps of
// 128 dealt round to its waves, whose sums are added in LDS in the waves' order.
// A step is requested while the one before is multiplied.  Bound by the codes' reading
// (16 x 37888 x 3584 at groups of 64: 19.6 us, 3.8 TB/s; 1 x 4096 x 4096: 4.5 us, of
// which a launch that does nothing takes about 2.5).
// GROUP: 32, 64 or 128 (a multiple of 128 applies one scale to several steps).
// In a fragment lane 16 j + r has the 32 codes of input group j of weight row r; a
// matrix instruction takes all its inputs from one such group instead, so that it
// never mixes scales: four lane-row exchanges per 32 codes.
template <int TM, int NG, int GROUP>
__global__ __launch_bounds__(TM == 4 ? 256 : 512) void w4a16_kernel(const uint16_t* __restrict__ X,
                                                                    const uint8_t* __restrict__ Wf,
                                                                    const uint16_t* __restrict__ s_w, int M, int N,
                                                                    int K, int group, uint16_t* __restrict__ Y) {
    extern __shared__ __attribute__((aligned(16))) uint8_t sm[];
    constexpr int CH = 128 / GROUP, PER = 4 / CH;      // scales a step, matrix instructions a scale
    const int waves = blockDim.x / kWave;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r = lane % 16, g = lane / 16;
    const int groups = (N + 15) / 16, steps = (K + 127) / 128;
    const int g0 = blockIdx.x * NG, m0 = blockIdx.y * (16 * TM);
    // Buffer loads: what lies past the last step, output or row reads as zero without
    // touching memory, and every step issues the same loads, so that waiting for one step's
    // leaves the next one's in flight.
    const __amdgpu_buffer_rsrc_t rW = make_rsrc(Wf, (uint32_t)groups * steps * 1024);
    const __amdgpu_buffer_rsrc_t rS = make_rsrc(s_w, (uint32_t)(K / group) * N * 2);
    const __amdgpu_buffer_rsrc_t rX = make_rsrc(X + (int64_t)m0 * K, (uint32_t)min(M - m0, 16 * TM) * K * 2);
    const int s_col = (g0 + r % NG) * 16 + 4 * g;
    const uint32_t sv = s_col < N ? (uint32_t)s_col * 2 : kOOB;
    uint32_t wv[NG], xv[TM];
#pragma unroll
    for (int n = 0; n < NG; ++n) wv[n] = g0 + n < groups ? (uint32_t)(g0 + n) * 1024 + lane * 16 : kOOB;
#pragma unroll
    for (int i = 0; i < TM; ++i) xv[i] = m0 + 16 * i + r < M ? (uint32_t)((16 * i + r) * K + 8 * g) * 2 : kOOB;
    // EDGE: the step may lie past the last one or be its half (K is a multiple of 64)
    auto fetch = [&](int t, auto edge, Step<TM, NG, CH>& f) {
        constexpr bool kEdge = decltype(edge)::value;
        const int at = kEdge ? min(t, steps - 1) : t;
        const bool in = !kEdge || t < steps;
#pragma unroll
        for (int n = 0; n < NG; ++n)
            f.w[n] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(rW, (int)(in ? wv[n] : kOOB),
                                                                                  at * groups * 1024, 0));
#pragma unroll
        for (int z = 0; z < CH; ++z) {
            int sg = GROUP < 128 ? at * CH + z : at / (group / 128);
            if (kEdge) sg = min(sg, K / group - 1);
            f.s[z] = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(rS, (int)(in ? sv : kOOB),
                                                                                   (int)((uint32_t)sg * N * 2), 0));
        }
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                // (an offset in the scalar part that passes the buffer would undo the check of the other)
                const bool some = !kEdge || t * 128 + 32 * s < K;
                f.x[i][s] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(
                                rX, (int)(some ? xv[i] : kOOB), some ? t * 256 + 64 * s : 0, 0));
            }
    };
    const NibbleMasks masks = nibble_masks();
    f4 sum[NG][TM];
#pragma unroll
    for (int n = 0; n < NG; ++n)
#pragma unroll
        for (int i = 0; i < TM; ++i) sum[n][i] = f4{0, 0, 0, 0};
    auto multiply = [&](const Step<TM, NG, CH>& f) {
        h8 x[TM][4];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int s = 0; s < 4; ++s) x[i][s] = same_order(f.x[i][s]);
        auto one = [&](auto index) {
            constexpr int n = decltype(index)::value;
            uint32_t c[4] = {(uint32_t)f.w[n][0], (uint32_t)f.w[n][1], (uint32_t)f.w[n][2], (uint32_t)f.w[n][3]};
            transpose_rows4(c[0], c[1], c[2], c[3]);
            h8 q[4];
#pragma unroll
            for (int s = 0; s < 4; ++s) q[s] = nibbles_to_halves(c[s], masks);
#pragma unroll
            for (int z = 0; z < CH; ++z) {
                const uint32_t s0 = row_broadcast<n>(f.s[z].x), s1 = row_broadcast<n>(f.s[z].y);
                const f4 sc{lo_h(s0), hi_h(s0), lo_h(s1), hi_h(s1)};
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    f4 acc{0, 0, 0, 0};
#pragma unroll
                    for (int s = z * PER; s < (z + 1) * PER; ++s)
                        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(q[s], x[i][s], acc, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[n][i][e] = __builtin_fmaf(acc[e], sc[e], sum[n][i][e]);
                }
            }
        };
        one(Index<0>());
        if constexpr (NG > 1) one(Index<1>());
        if constexpr (NG > 2) one(Index<2>());
        if constexpr (NG > 3) one(Index<3>());
        if constexpr (NG > 4) one(Index<4>());
    };
    if (wave < steps) {
        // all but the last two steps of a wave lie inside; past the last, zeros are read and
        // nothing is multiplied
        Step<TM, NG, CH> a, b;
        fetch(wave, Index<1>(), a);
        int t = wave;
        for (; t + 2 * waves < steps - 1; t += 2 * waves) {
            fetch(t + waves, Index<0>(), b);
            multiply(a);
            fetch(t + 2 * waves, Index<0>(), a);
            multiply(b);
        }
        for (;; t += 2 * waves) {
            fetch(t + waves, Index<1>(), b);
            multiply(a);
            if (t + waves >= steps) break;
            fetch(t + 2 * waves, Index<1>(), a);
            multiply(b);
            if (t + 2 * waves >= steps) break;
        }
    }
    f4* red = reinterpret_cast<f4*>(sm);               // [wave][NG][TM][lane]
#pragma unroll
    for (int n = 0; n < NG; ++n)
#pragma unroll
        for (int i = 0; i < TM; ++i) red[((wave * NG + n) * TM + i) * kWave + lane] = sum[n][i];
    __syncthreads();
    // the waves share the adding up: of the NG TM tiles, number z to wave z % waves
    for (int z = wave; z < NG * TM; z += waves) {
        const int n = z / TM, i = z % TM;
        f4 y = red[z * kWave + lane];
        for (int v = 1; v < waves; ++v) y += red[(v * NG * TM + z) * kWave + lane];
        const int m = m0 + 16 * i + r, o = (g0 + n) * 16 + 4 * g;
        if (m < M && o < N) {
            uint2 w;
            w.x = (uint32_t)f2h(y[0]) | ((uint32_t)f2h(y[1]) << 16);
            w.y = (uint32_t)f2h(y[2]) | ((uint32_t)f2h(y[3]) << 16);
            *reinterpret_cast<uint2*>(Y + (int64_t)m * N + o) = w;
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
    float m = 0.0f;                                    // NaN if a weight is
    for (int e = lane; e < group / 2; e += kWave)
        m = __builtin_elementwise_maximum(m, __builtin_elementwise_maximum(fabsf(lo_h(w[e])), fabsf(hi_h(w[e]))));
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) m = __builtin_elementwise_maximum(m, __shfl_xor(m, o, kWave));
    const uint16_t sh = f2h(m / 7.0f);
    const float s = h2f(sh);
    const bool some = s > 0.0f && s < __builtin_inff();
    uint8_t* q = Wq + ((int64_t)n * K + gi * group) / 2;
    for (int e = lane; e < group / 2; e += kWave) {
        const int a = some ? quant4(lo_h(w[e]), s) : 0, b = some ? quant4(hi_h(w[e]), s) : 0;
        q[e] = (uint8_t)((a & 15) | ((b & 15) << 4));
    }
    if (lane == 0) s_w[(int64_t)gi * N + n] = sh;
}

template <int TM, int NG>
hipError_t launch_tile(const uint16_t* X, const uint8_t* Wf, const uint16_t* s_w, int M, int N, int K, int group,
                       uint16_t* Y, int waves, hipStream_t st) {
    const dim3 grid((unsigned)(((N + 15) / 16 + NG - 1) / NG), (unsigned)((M + 16 * TM - 1) / (16 * TM)));
    const dim3 block(kWave * waves);
    const size_t lds = (size_t)waves * NG * TM * kWave * sizeof(f4);
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
    const W4a16Plan p = w4a16_plan(M, N);
    switch (p.tm * 8 + p.ng) {
        case 8 + 1: return launch_tile<1, 1>(X, Wf, s_w, M, N, K, group, Y, p.waves, st);
        case 8 + 2: return launch_tile<1, 2>(X, Wf, s_w, M, N, K, group, Y, p.waves, st);
        case 8 + 3: return launch_tile<1, 3>(X, Wf, s_w, M, N, K, group, Y, p.waves, st);
        case 8 + 4: return launch_tile<1, 4>(X, Wf, s_w, M, N, K, group, Y, p.waves, st);
        case 8 + 5: return launch_tile<1, 5>(X, Wf, s_w, M, N, K, group, Y, p.waves, st);
        case 16 + 1: return launch_tile<2, 1>(X, Wf, s_w, M, N, K, group, Y, p.waves, st);
        case 16 + 2: return launch_tile<2, 2>(X, Wf, s_w, M, N, K, group, Y, p.waves, st);
        case 32 + 1: return launch_tile<4, 1>(X, Wf, s_w, M, N, K, group, Y, p.waves, st);
        case 32 + 2: return launch_tile<4, 2>(X, Wf, s_w, M, N, K, group, Y, p.waves, st);
        default: return hipErrorInvalidConfiguration;
    }
}

}  // namespace sq
