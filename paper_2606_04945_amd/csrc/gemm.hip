// Products on row-major weights and the reordering of weights; the kernels they share with the
// fragment-ordered products, and how codes become operands, are in gemm_kernels.hpp.
#include "gemm_kernels.hpp"
#include "layer.hpp"

namespace sq {
namespace {

// KW waves share one group of 16 columns and take turns over k, batch by batch
// (wave w multiplies batches w, w + KW, ...); their partial sums meet in LDS.
// Activation fragments come from global memory (they stay in L2: every
// workgroup reads the same M x K codes).  The K split gives narrow layers
// enough waves to keep HBM busy.
template <int U, int KW, int TM, int BITS>
__global__ __launch_bounds__(64 * KW) void gemm_skinny_kernel(const uint8_t* __restrict__ Aq,
                                                              const float* __restrict__ s_a,
                                                              const uint8_t* __restrict__ Wq,
                                                              const float* __restrict__ s_w, int M, int N, int K,
                                                              uint16_t* __restrict__ Y, int32_t* __restrict__ acc_out) {
    constexpr int D = 2;
    __shared__ v4i red[KW > 1 ? KW - 1 : 1][TM][kWave];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int lr = lane % 16, lg = lane / 16;
    const int col = blockIdx.x * 16 + lr;
    const uint32_t ldb = (uint32_t)K * BITS / 8;
    const int nk = (int)((ldb + kKB - 1) / kKB);
    const int nb = (nk + U - 1) / U;
    const __amdgpu_buffer_rsrc_t rA = make_rsrc(Aq, (uint32_t)M * ldb);
    const __amdgpu_buffer_rsrc_t rW = make_rsrc(Wq, (uint32_t)N * ldb);
    const uint32_t seg = 16 * lg;
    const uint32_t ow = (uint32_t)min(col, N - 1) * ldb + seg;
    uint32_t oa[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) oa[i] = (uint32_t)min(16 * i + lr, M - 1) * ldb + seg;
    const uint32_t alim = ldb > seg ? ldb - seg : 0;   // this lane's activation bytes end here
    auto issue = [&](int b, v4i (&w)[U], v4i (&a)[U][TM]) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int kt = b * U + u;
            const int so = step_offset(kt, nk);
            const bool in = (uint32_t)kt * kKB < alim;
            w[u] = __builtin_amdgcn_raw_buffer_load_b128(rW, (int)ow, so, 0);
#pragma unroll
            for (int i = 0; i < TM; ++i)
                a[u][i] = __builtin_amdgcn_raw_buffer_load_b128(rA, in ? (int)oa[i] : (int)kOOB, so, 0);
        }
    };
    v4i acc[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) acc[i] = v4i{0, 0, 0, 0};
    auto compute = [&](const v4i (&w)[U], const v4i (&a)[U][TM]) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < (BITS == 4 ? 2 : 1); ++h) {
                const v4i wop = operand<BITS>(w[u], h);
#pragma unroll
                for (int i = 0; i < TM; ++i)
                    acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(operand<BITS>(a[u][i], h), wop, acc[i], 0, 0, 0);
            }
    };
    v4i w[D][U], a[D][U][TM];
    issue(wave, w[0], a[0]);
    float sav[TM][4];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) sav[i][r] = s_a[min(16 * i + 4 * lg + r, M - 1)];
    const float swv = s_w[min(col, N - 1)];
    int b = wave;
    do {
        issue(b + KW, w[1], a[1]);
        __builtin_amdgcn_sched_barrier(0);
        compute(w[0], a[0]);
        __builtin_amdgcn_sched_barrier(0);
        issue(b + 2 * KW, w[0], a[0]);
        __builtin_amdgcn_sched_barrier(0);
        compute(w[1], a[1]);
        __builtin_amdgcn_sched_barrier(0);
        b += 2 * KW;
    } while (b < nb);
    if (KW > 1) {
        if (wave > 0) {
#pragma unroll
            for (int i = 0; i < TM; ++i) red[wave - 1][i][lane] = acc[i];
        }
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int r = 0; r < KW - 1; ++r)
#pragma unroll
            for (int i = 0; i < TM; ++i) acc[i] += red[r][i][lane];
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) skinny_store<BITS>(acc[i], 16 * i, lg, col, M, N, sav[i], swv, Y, acc_out);
}

// Wide layers, 4-bit codes: the workgroup's waves (blockDim.x / 64 of them)
// each stream their own 16 columns, and the M x K activation codes are staged
// once per workgroup in LDS by a direct-to-LDS copy (zero past M and K), instead
// of being fetched by every wave.  With one row tile (M <= 16) they are then
// expanded once, by all waves together, to MFMA operands ([k step][half][lane]
// [16 B]); with more row tiles each wave expands its fragments as it multiplies
// (the expanded copy would not fit).  The weight ring is issued before the copy
// is waited on, so the first batches are already in flight.
constexpr int kSharedU = 2, kSharedD = 4;

template <int TM>
__global__ __launch_bounds__(64 * kSharedMaxWaves) void gemm_skinny_shared_kernel(
    const uint8_t* __restrict__ Aq, const float* __restrict__ s_a, const uint8_t* __restrict__ Wq,
    const float* __restrict__ s_w, int M, int N, int K, uint16_t* __restrict__ Y, int32_t* __restrict__ acc_out) {
    constexpr int U = kSharedU, D = kSharedD;
    constexpr bool kExpand = TM == 1;
    extern __shared__ __attribute__((aligned(16))) uint8_t sm[];
    const int nw = blockDim.x / kWave;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int lr = lane % 16, lg = lane / 16;
    const int col = (blockIdx.x * nw + wave) * 16 + lr;
    const uint32_t ldb = (uint32_t)K / 2;
    const int nk = (int)((ldb + kKB - 1) / kKB);
    const int nb = (nk + U - 1) / U;
    uint8_t* raw = sm;                   // [TM][nk] x 1 KB: packed activation fragments
    uint8_t* ops = sm + nk * 1024;       // one row tile: nk x 2 KB of expanded operands
    const u32x4 rA = sgpr_rsrc(Aq, (uint32_t)M * ldb);
    const __amdgpu_buffer_rsrc_t rW = make_rsrc(Wq, (uint32_t)N * ldb);
    const uint32_t seg = 16 * lg;
    for (int p = wave; p < TM * nk; p += nw) {
        const int row = 16 * (p / nk) + lr;
        const uint32_t ko = (uint32_t)(p % nk) * kKB;
        dma16(rA, lds_addr(raw + p * 1024), (row < M && ko + seg < ldb) ? (uint32_t)row * ldb + ko + seg : kOOB);
    }
    const uint32_t ow = (uint32_t)min(col, N - 1) * ldb + seg;
    auto issue = [&](int b, v4i (&w)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            w[u] = __builtin_amdgcn_raw_buffer_load_b128(rW, (int)ow, step_offset(b * U + u, nk), 0);
    };
    v4i w[D][U];
#pragma unroll
    for (int d = 0; d < D - 1; ++d) issue(d, w[d]);
    wait_vm<(D - 1) * U>();              // this wave's copies have landed (its weight loads may not have)
    __builtin_amdgcn_s_barrier();        // ... and every wave's
    asm volatile("" ::: "memory");
    if (kExpand) {
        for (int s = wave; s < nk; s += nw) {
            const v4i r = *reinterpret_cast<const v4i*>(raw + s * 1024 + lane * 16);
            *reinterpret_cast<v4i*>(ops + (2 * s) * 1024 + lane * 16) = operand<4>(r, 0);
            *reinterpret_cast<v4i*>(ops + (2 * s + 1) * 1024 + lane * 16) = operand<4>(r, 1);
        }
        __syncthreads();
    }
    float sav[TM][4];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) sav[i][r] = s_a[min(16 * i + 4 * lg + r, M - 1)];
    const float swv = s_w[min(col, N - 1)];
    v4i acc[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) acc[i] = v4i{0, 0, 0, 0};
    auto compute = [&](int b, const v4i (&wb)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int kt = min(b * U + u, nk - 1);      // past the end the weights read as zero
            v4i ar[TM];
            if (!kExpand) {
#pragma unroll
                for (int i = 0; i < TM; ++i) ar[i] = *reinterpret_cast<const v4i*>(raw + (i * nk + kt) * 1024 + lane * 16);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const v4i wop = operand<4>(wb[u], h);
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    const v4i x = kExpand ? *reinterpret_cast<const v4i*>(ops + (2 * kt + h) * 1024 + lane * 16)
                                          : operand<4>(ar[i], h);
                    acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x, wop, acc[i], 0, 0, 0);
                }
            }
        }
    };
    int b = 0;
    do {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            issue(b + d + D - 1, w[(d + D - 1) % D]);
            __builtin_amdgcn_sched_barrier(0);
            compute(b + d, w[d]);
            __builtin_amdgcn_sched_barrier(0);
        }
        b += D;
    } while (b < nb);
#pragma unroll
    for (int i = 0; i < TM; ++i) skinny_store<4>(acc[i], 16 * i, lg, col, M, N, sav[i], swv, Y, acc_out);
}

// Packed int4 weights [N][K/2] -> fragment order: one thread per 16-byte unit
// (k step t, group g, lane l) = bytes 64 t + 16 (l / 16) .. + 15 of row
// 16 g + l % 16, zero past N and past the row.  Gated: rows [gates, ups] of N / 2 each; group g
// takes gates 8 g .. + 7, then their ups.
__global__ __launch_bounds__(256) void weights_to_frag_kernel(const uint8_t* __restrict__ Wq, int N, int K, bool glu,
                                                              uint8_t* __restrict__ Wf) {
    const uint32_t ldb = (uint32_t)K / 2;
    const uint32_t nk = (ldb + kKB - 1) / kKB;
    const uint32_t ngrp = (uint32_t)(N + 15) / 16;
    const size_t units = (size_t)ngrp * nk * kWave;
    for (size_t e = (size_t)blockIdx.x * 256 + threadIdx.x; e < units; e += (size_t)gridDim.x * 256) {
        const uint32_t l = (uint32_t)(e % kWave);
        const size_t tg = e / kWave;
        const uint32_t g = (uint32_t)(tg % ngrp), t = (uint32_t)(tg / ngrp);
        const uint32_t r = l % 16, byte = t * kKB + 16 * (l / 16);
        const uint32_t row = glu ? 8 * g + r % 8 + (r / 8) * ((uint32_t)N / 2) : 16 * g + r;
        v4i v = v4i{0, 0, 0, 0};
        if (row < (uint32_t)N && byte < ldb) v = *reinterpret_cast<const v4i*>(Wq + (size_t)row * ldb + byte);
        *reinterpret_cast<v4i*>(Wf + e * 16) = v;
    }
}

template <int U, int KW, int TM, int BITS>
hipError_t launch_skinny(const uint8_t* Aq, const float* s_a, const uint8_t* Wq, const float* s_w, int M, int N,
                         int K, uint16_t* Y, int32_t* acc, hipStream_t st) {
    hipLaunchKernelGGL((gemm_skinny_kernel<U, KW, TM, BITS>), dim3((N + 15) / 16), dim3(64 * KW), 0, st, Aq, s_a, Wq,
                       s_w, M, N, K, Y, acc);
    return hipGetLastError();
}

template <int TM>
hipError_t launch_skinny_shared_tm(int waves, const uint8_t* Aq, const float* s_a, const uint8_t* Wq,
                                   const float* s_w, int M, int N, int K, uint16_t* Y, int32_t* acc, hipStream_t st) {
    const int nk = (K / 2 + kKB - 1) / kKB;
    const size_t lds = shared_lds_bytes(TM, nk);
    static std::atomic<int> lds_set[kMaxDevices];   // above the 64 KB default for dynamic LDS
    const hipError_t attr =
        allow_dynamic_lds(reinterpret_cast<const void*>(&gemm_skinny_shared_kernel<TM>),
                          (int)(TM == 1 ? kSharedMaxSteps * 3 * 1024 : kSharedMaxTileSteps * 1024), lds_set);
    if (attr != hipSuccess) return attr;
    if (lds == 0 || waves < 1 || waves > kSharedMaxWaves) return hipErrorInvalidConfiguration;
    const int groups = (N + 15) / 16;
    hipLaunchKernelGGL((gemm_skinny_shared_kernel<TM>), dim3((groups + waves - 1) / waves), dim3(64 * waves), lds,
                       st, Aq, s_a, Wq, s_w, M, N, K, Y, acc);
    return hipGetLastError();
}

hipError_t launch_skinny_shared(int waves, const uint8_t* Aq, const float* s_a, const uint8_t* Wq, const float* s_w,
                                int M, int N, int K, uint16_t* Y, int32_t* acc, hipStream_t st) {
    switch ((M + 15) / 16) {
        case 1: return launch_skinny_shared_tm<1>(waves, Aq, s_a, Wq, s_w, M, N, K, Y, acc, st);
        case 2: return launch_skinny_shared_tm<2>(waves, Aq, s_a, Wq, s_w, M, N, K, Y, acc, st);
        case 3: return launch_skinny_shared_tm<3>(waves, Aq, s_a, Wq, s_w, M, N, K, Y, acc, st);
        default: return hipErrorInvalidConfiguration;
    }
}

template <int TM, int BITS>
hipError_t skinny_kw_tm(int kw, const uint8_t* Aq, const float* s_a, const uint8_t* Wq, const float* s_w, int M, int N,
                        int K, uint16_t* Y, int32_t* acc, hipStream_t st) {
    // two register batches of U k steps in flight: 8 steps per batch for one row
    // tile and up to two waves per column group, 4 for four or eight waves, 2 for
    // more row tiles (each step holds TM + 1 fragments)
    constexpr int U1 = TM == 1 ? 8 : 2, U4 = TM == 1 ? 4 : 2;
    switch (kw) {
        case 1: return launch_skinny<U1, 1, TM, BITS>(Aq, s_a, Wq, s_w, M, N, K, Y, acc, st);
        case 2: return launch_skinny<U1, 2, TM, BITS>(Aq, s_a, Wq, s_w, M, N, K, Y, acc, st);
        case 4: return launch_skinny<U4, 4, TM, BITS>(Aq, s_a, Wq, s_w, M, N, K, Y, acc, st);
        default: return launch_skinny<U4, 8, TM, BITS>(Aq, s_a, Wq, s_w, M, N, K, Y, acc, st);
    }
}

template <int BITS>
hipError_t skinny_kw(int kw, const uint8_t* Aq, const float* s_a, const uint8_t* Wq, const float* s_w, int M, int N,
                     int K, uint16_t* Y, int32_t* acc, hipStream_t st) {
    switch ((M + 15) / 16) {
        case 1: return skinny_kw_tm<1, BITS>(kw, Aq, s_a, Wq, s_w, M, N, K, Y, acc, st);
        case 2: return skinny_kw_tm<2, BITS>(kw, Aq, s_a, Wq, s_w, M, N, K, Y, acc, st);
        case 3: return skinny_kw_tm<3, BITS>(kw, Aq, s_a, Wq, s_w, M, N, K, Y, acc, st);
        default: return hipErrorInvalidConfiguration;
    }
}

}  // namespace

size_t frag_weight_bytes(int N, int K) {
    return (size_t)((N + 15) / 16) * (size_t)((K / 2 + kKB - 1) / kKB) * 1024;
}

static hipError_t to_frag(const uint8_t* Wq, int N, int K, uint8_t* Wf, hipStream_t st, bool glu) {
    const size_t units = frag_weight_bytes(N, K) / 16;
    const size_t blocks = (units + 255) / 256;
    hipLaunchKernelGGL(weights_to_frag_kernel, dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, st, Wq,
                       N, K, glu, Wf);
    return hipGetLastError();
}

hipError_t launch_weights_to_frag(const uint8_t* Wq, int N, int K, uint8_t* Wf, hipStream_t st) {
    return to_frag(Wq, N, K, Wf, st, false);
}

hipError_t launch_weights_to_frag_glu(const uint8_t* Wq, int N, int K, uint8_t* Wf, hipStream_t st) {
    return to_frag(Wq, N, K, Wf, st, true);
}

hipError_t launch_gemm_frag(const uint8_t* Aq, const float* s_a, const uint8_t* Wf, const float* s_w, int M, int N,
                            int K, uint16_t* Y, int32_t* acc, void* ws, hipStream_t st, int bits) {
    return run_frag(Aq, s_a, Wf, s_w, M, N, K, Y, acc, ws, st, bits, Dequant{});
}

size_t gemm_workspace_bytes(int M, int N, int K, int bits) { return plan_workspace_bytes(M, N, K, bits); }

hipError_t launch_gemm(const uint8_t* Aq, const float* s_a, const uint8_t* Wq, const float* s_w, int M, int N,
                       int K, uint16_t* Y, int32_t* acc, void* ws, hipStream_t st, int bits) {
    const Plan p = gemm_plan(M, N, K, bits, false);
    int32_t* part = static_cast<int32_t*>(ws);
    hipError_t e;
    if (bits == 8) {
        switch (p.cfg) {
            case 3: e = skinny_kw<8>(p.waves, Aq, s_a, Wq, s_w, M, N, K, Y, acc, st); break;
            case 7: e = launch_tiled<2, 2, 4, 8, 8, 2>(p, Aq, s_a, Wq, s_w, M, N, K, Y, acc, part, st); break;
            case 9: e = launch_tiled<2, 2, 4, 4, 8, 2, false, 2>(p, Aq, s_a, Wq, s_w, M, N, K, Y, acc, part, st); break;
            case 10: e = launch_tiled<1, 1, 2, 2, 8, 3, false, 12>(p, Aq, s_a, Wq, s_w, M, N, K, Y, acc, part, st); break;
            case 11: e = launch_tiled<1, 2, 2, 2, 8, 4, false, 8>(p, Aq, s_a, Wq, s_w, M, N, K, Y, acc, part, st); break;
            case 12: e = launch_tiled<2, 1, 2, 4, 8, 2, false, 4>(p, Aq, s_a, Wq, s_w, M, N, K, Y, acc, part, st); break;
            case 13: e = launch_tiled<2, 2, 2, 4, 8, 2, false, 2>(p, Aq, s_a, Wq, s_w, M, N, K, Y, acc, part, st); break;
            case 14: e = launch_tiled<1, 4, 4, 2, 8, 2, false, 3>(p, Aq, s_a, Wq, s_w, M, N, K, Y, acc, part, st); break;
            case 8: e = launch_tiled<1, 2, 8, 4, 8, 2>(p, Aq, s_a, Wq, s_w, M, N, K, Y, acc, part, st); break;
            case 1: e = launch_tiled<2, 2, 4, 4, 8, 3>(p, Aq, s_a, Wq, s_w, M, N, K, Y, acc, part, st); break;
            case 2: e = launch_tiled<2, 2, 2, 2, 8, 4>(p, Aq, s_a, Wq, s_w, M, N, K, Y, acc, part, st); break;
            default: return hipErrorInvalidConfiguration;
        }
    } else {
        switch (p.cfg) {
            case 3: e = skinny_kw<4>(p.waves, Aq, s_a, Wq, s_w, M, N, K, Y, acc, st); break;
            case 5: e = launch_skinny_shared(p.waves, Aq, s_a, Wq, s_w, M, N, K, Y, acc, st); break;
            case 0: e = launch_tiled<4, 2, 4, 4, 4, 2>(p, Aq, s_a, Wq, s_w, M, N, K, Y, acc, part, st); break;
            case 9: e = launch_tiled<2, 2, 4, 4, 4, 2, false, 2>(p, Aq, s_a, Wq, s_w, M, N, K, Y, acc, part, st); break;
            case 10: e = launch_tiled<1, 1, 2, 2, 4, 3, false, 12>(p, Aq, s_a, Wq, s_w, M, N, K, Y, acc, part, st); break;
            case 11: e = launch_tiled<1, 2, 2, 2, 4, 4, false, 8>(p, Aq, s_a, Wq, s_w, M, N, K, Y, acc, part, st); break;
            case 12: e = launch_tiled<2, 1, 2, 4, 4, 2, false, 4>(p, Aq, s_a, Wq, s_w, M, N, K, Y, acc, part, st); break;
            case 13: e = launch_tiled<2, 2, 2, 4, 4, 2, false, 2>(p, Aq, s_a, Wq, s_w, M, N, K, Y, acc, part, st); break;
            case 14: e = launch_tiled<1, 4, 4, 2, 4, 2, false, 3>(p, Aq, s_a, Wq, s_w, M, N, K, Y, acc, part, st); break;
            case 1: e = launch_tiled<2, 2, 4, 4, 4, 3>(p, Aq, s_a, Wq, s_w, M, N, K, Y, acc, part, st); break;
            case 2: e = launch_tiled<2, 2, 2, 2, 4, 4>(p, Aq, s_a, Wq, s_w, M, N, K, Y, acc, part, st); break;
            case 4: e = launch_tiled<1, 4, 4, 2, 4, 4>(p, Aq, s_a, Wq, s_w, M, N, K, Y, acc, part, st); break;
            default: return hipErrorInvalidConfiguration;
        }
    }
    if (e != hipSuccess) return e;
    return finish_split(p, part, s_a, s_w, M, N, Y, acc, st);
}

}  // namespace sq
