// Attention over the paged 8-bit cache for few rows: every load goes straight to
// registers and no wave waits for another inside the loop over keys.
//
// The matrix instruction is 16 x 16 x 32.  Matrix row c of key tile s is key
// 16 (c / 4) + 4 s + c % 4 of the step, so lane group g's four accumulators hold keys
// 16 g .. 16 g + 15, and it reads its values as 16 contiguous bytes a channel; keys
// are read as 16 contiguous channels.  A lane group's keys share a page, and with it
// one pair of scales.
#include "attn_common.hpp"

namespace sq {
namespace {

// over the four 16-lane groups of a wave
__device__ __forceinline__ float groups_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16, kWave));
    return fmaxf(x, __shfl_xor(x, 32, kWave));
}
__device__ __forceinline__ float groups_sum(float x) {
    x += __shfl_xor(x, 16, kWave);
    return x + __shfl_xor(x, 32, kWave);
}

// One wave's rows of a tile: 16 QT of them, and the pass over some of their steps.
// DP: head size rounded up to 64, 128 or 256.
template <int DP, int QT>
struct WaveRows {
    static constexpr int P = DP / 64, DT = DP / 16;
    int t[QT], qh[QT], lo[QT], hi[QT];    // batch row, query head, visible keys of this lane's column
    bool in[QT];
    h8 Q[QT][2 * P];
    f4 O[QT][DT];
    float m[QT], l[QT];

    __device__ __forceinline__ void begin(const AttnArgs& p, const Seq& s, int h, int r, int c, int g) {
        const int G = p.a.G, rows = s.n * G;
#pragma unroll
        for (int y = 0; y < QT; ++y) {
            const int row = r * (16 * QT) + 16 * y + c;
            in[y] = row < rows;
            const int at = min(row, rows - 1), i = at / G;
            t[y] = s.t0 + i;
            qh[y] = h * G + at % G;
            lo[y] = attn_lo(p.a, s.off + i);
            hi[y] = attn_hi(p.a, s, s.off + i);
            const uint16_t* q = p.Q + t[y] * p.q_token + qh[y] * p.q_head;
#pragma unroll
            for (int z = 0; z < 2 * P; ++z) {
                const int d = 64 * (z / 2) + 16 * g + 8 * (z % 2);
                Q[y][z] = d < p.D ? load_query(q + d, p.flip) : h8{};
            }
            m[y] = kUnseen, l[y] = 0.0f;
#pragma unroll
            for (int d = 0; d < DT; ++d) O[y][d] = f4{0, 0, 0, 0};
        }
    }

    // Steps first, first + stride, ... below end.  What the next step reads is
    // requested as soon as the registers of this one's are free: its keys before this
    // step's softmax, its values after the second product, its pages a step earlier.
    __device__ __forceinline__ void pass(const AttnArgs& p, const Seq& s, int b, int h, int first, int end, int stride,
                                         int c, int g) {
        if (first >= end) return;
        const int32_t* table = p.table + (int64_t)b * p.max_pages;
        const int D = p.D;
        int kp, vp, kn, vn;                       // pages of this lane's key row and of its lane group, now and next
        auto pages = [&](int kt, int& a, int& z) {
            const int ka = kt * kAttnStep + 16 * (c / 4), va = kt * kAttnStep + 16 * g;
            a = ka < s.len ? table[ka >> p.shift] : -1;
            z = va < s.len ? table[va >> p.shift] : -1;
        };
        v4i kw[4][P], vw[DT];
        float ks, vs;
        auto keys = [&](int kt, int pid) {
            const int ka = kt * kAttnStep + 16 * (c / 4);
            const int64_t ph = (uint32_t)pid < (uint32_t)p.pages ? (int64_t)pid * p.a.heads + h : h;
            const int8_t* at = p.k + (ph * p.page + (ka & (p.page - 1)) + c % 4) * D + 16 * g;
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int z = 0; z < P; ++z)
                    kw[e][z] = 64 * z + 16 * g < D ? *reinterpret_cast<const v4i*>(at + 4 * e * D + 64 * z)
                                                   : v4i{0, 0, 0, 0};
        };
        auto values = [&](int kt, int pid) {
            const int va = kt * kAttnStep + 16 * g;
            const int64_t ph = (uint32_t)pid < (uint32_t)p.pages ? (int64_t)pid * p.a.heads + h : h;
            const int8_t* at = p.v + ph * p.page * D + (va & (p.page - 1));
#pragma unroll
            for (int d = 0; d < DT; ++d) vw[d] = *reinterpret_cast<const v4i*>(at + min(16 * d + c, D - 1) * p.page);
        };
        auto scales = [&](int pid) {
            const int64_t ph = (uint32_t)pid < (uint32_t)p.pages ? (int64_t)pid * p.a.heads + h : h;
            ks = p.k_scale[ph];
            vs = p.v_scale[ph];
        };
        pages(first, kp, vp);
        kn = vn = -1;
        if (first + stride < end) pages(first + stride, kn, vn);
        keys(first, kp);
        scales(vp);
        values(first, vp);
        for (int kt = first; kt < end; kt += stride) {
            const bool more = kt + stride < end;
            const int key0 = kt * kAttnStep, va = key0 + 16 * g;
            const bool vin = (uint32_t)vp < (uint32_t)p.pages;
            f4 S[QT][4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
#pragma unroll
                for (int y = 0; y < QT; ++y) S[y][e] = f4{0, 0, 0, 0};
#pragma unroll
                for (int z = 0; z < 2 * P; ++z) {
                    const v4i w = kw[e][z / 2];
                    const h8 k = to_halves((uint32_t)w[2 * (z % 2)], (uint32_t)w[2 * (z % 2) + 1]);
#pragma unroll
                    for (int y = 0; y < QT; ++y)
                        S[y][e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, Q[y][z], S[y][e], 0, 0, 0);
                }
            }
            const float ks0 = ks, vs0 = vs;
            if (more) {
                kp = kn, vp = vn;
                keys(kt + stride, kp);
                scales(vp);
                kn = vn = -1;
                if (kt + 2 * stride < end) pages(kt + 2 * stride, kn, vn);
            }
            h8 W[QT][2];
#pragma unroll
            for (int y = 0; y < QT; ++y) {
                const BlockScale bs = block_scale(vin, ks0, vs0, p.scale);
                if (!__all(key0 >= lo[y] && key0 + kAttnStep <= hi[y])) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int key = va + 4 * e + i;
                            if (key < lo[y] || key >= hi[y]) S[y][e][i] = kHidden;
                        }
                }
                float mx = S[y][0][0];
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int i = 0; i < 4; ++i) mx = fmaxf(mx, S[y][e][i]);
                mx = fmaxf(m[y], groups_max(__builtin_fmaf(mx, bs.ks, bs.lv)));
                const float fade = __builtin_amdgcn_exp2f(m[y] - mx), off = bs.lv - mx;
                m[y] = mx;
                float sum = 0.0f;
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int i = 0; i < 4; i += 2) {
                        const f2 w = {__builtin_amdgcn_exp2f(__builtin_fmaf(S[y][e][i], bs.ks, off)),
                                      __builtin_amdgcn_exp2f(__builtin_fmaf(S[y][e][i + 1], bs.ks, off))};
                        sum += w[0];
                        sum += w[1];
                        const h2 x = __builtin_convertvector(w, h2);
                        W[y][e / 2][4 * (e % 2) + i] = x[0];
                        W[y][e / 2][4 * (e % 2) + i + 1] = x[1];
                    }
                l[y] = __builtin_fmaf(sum, bs.iv, l[y] * fade);
#pragma unroll
                for (int d = 0; d < DT; ++d) O[y][d] *= fade;
            }
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const h8 v = to_halves((uint32_t)vw[d][2 * u], (uint32_t)vw[d][2 * u + 1]);
#pragma unroll
                    for (int y = 0; y < QT; ++y)
                        O[y][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, W[y][u], O[y][d], 0, 0, 0);
                }
            if (more) values(kt + stride, vp);
        }
#pragma unroll
        for (int y = 0; y < QT; ++y) l[y] = groups_sum(l[y]);
    }

    __device__ __forceinline__ void store(const AttnArgs& p, int g) const {
#pragma unroll
        for (int y = 0; y < QT; ++y) {
            if (!in[y]) continue;
            const float inv = l[y] > 0.0f ? 1.0f / l[y] : 0.0f;
            const int64_t o = (int64_t)t[y] * p.a.heads * p.a.G + qh[y];
#pragma unroll
            for (int d = 0; d < DT; ++d)
                if (16 * d < p.D) store_result(p.O + o * p.D + 16 * d + 4 * g, O[y][d], inv);
            if (p.lse && g == 0) p.lse[o] = result_lse(m[y], l[y]);
        }
    }

    __device__ __forceinline__ void store_partial(const AttnArgs& p, float* ws, int c, int g) const {
        constexpr int R = 16 * QT;
#pragma unroll
        for (int y = 0; y < QT; ++y) {
            if (!in[y]) continue;
            const int row = 16 * y + c;
#pragma unroll
            for (int d = 0; d < DT; ++d)
                if (16 * d < p.D) *reinterpret_cast<f4*>(ws + row * p.D + 16 * d + 4 * g) = O[y][d];
            if (g == 0) ws[R * p.D + row] = m[y], ws[R * p.D + R + row] = l[y];
        }
    }
};

// Direct: a workgroup is a tile, whose steps go round its waves, and their results
// meet in LDS.  Otherwise every wave is a worker of the shared work.
template <int DP, int QT, int NW>
__global__ __launch_bounds__(NW* kWave) void attn_wave_kernel(AttnArgs p) {
    extern __shared__ __attribute__((aligned(16))) float lds[];
    constexpr int R = 16 * QT, LD = DP + 4;            // rows, padded row of floats
    float* ml = lds + NW * R * LD;                     // [wave][row] m, then l
    const int lane = threadIdx.x % kWave, c = lane % 16, g = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const Group first = load_group(p, 0, lane);
    const Survey all = survey(p, first, lane);
    Share sh{0, 0, 0, 0};
    Tile t{};
    int worker = 0, stride = 1, count = 0;
    if (all.direct) {
        const int64_t item = blockIdx.x / p.a.heads;
        const Listed at = find_listed<false>(p, item, first, lane);
        const int64_t r64 = item - list_start(at.q.s.t0, at.b, p.a.G, R, 1);
        if (r64 < 0 || r64 >= at.q.tiles) return;
        const AttnSteps steps = attn_steps(p.a, at.q.s, (int)r64);
        count = steps.count;
        stride = NW;
        t = {at.q.s, at.b, (int)(blockIdx.x % p.a.heads), (int)r64,
             {0, steps.first + wave, steps.first + steps.count, false, false}};
    } else {
        if ((int)blockIdx.x >= p.a.groups) return;
        worker = xcd_worker(blockIdx.x, p.a.groups) * NW + wave;
        sh = find_share(p, all.total, first, worker, lane);
    }
    for (;;) {
        if (!all.direct && !next_tile(p, sh, t)) return;
        WaveRows<DP, QT> w;
        w.begin(p, t.s, t.h, t.r, c, g);
        w.pass(p, t.s, t.b, t.h, t.part.k0, t.part.k1, stride, c, g);
        if (!all.direct) {
            if (t.part.whole)
                w.store(p, g);
            else
                w.store_partial(p, p.ws + attn_place(worker, t.part.inside) * attn_place_floats(R, p.D), c, g);
            continue;
        }
        const int waves = min(count, NW);              // those that had a step
        if (waves <= 1) {
            if (wave == 0) w.store(p, g);
            return;
        }
        if (wave < waves) {
#pragma unroll
            for (int y = 0; y < QT; ++y) {
                const int row = 16 * y + c;
#pragma unroll
                for (int d = 0; d < DP / 16; ++d)
                    if (16 * d < p.D) *reinterpret_cast<f4*>(lds + (wave * R + row) * LD + 16 * d + 4 * g) = w.O[y][d];
                if (g == 0) ml[wave * R + row] = w.m[y], ml[(NW + wave) * R + row] = w.l[y];
            }
        }
        __syncthreads();
        const int rows = min(R, t.s.n * p.a.G - t.r * R), vecs = p.D / 4;
        for (int e = threadIdx.x; e < rows * vecs; e += NW * kWave) {
            const int row = e / vecs, d = e % vecs * 4;
            float m = kUnseen;
            for (int v = 0; v < waves; ++v) m = fmaxf(m, ml[v * R + row]);
            float l = 0.0f;
            f4 O{0, 0, 0, 0};
            for (int v = 0; v < waves; ++v) {
                const float f = __builtin_amdgcn_exp2f(ml[v * R + row] - m);
                l = __builtin_fmaf(ml[(NW + v) * R + row], f, l);
                O += *reinterpret_cast<const f4*>(lds + (v * R + row) * LD + d) * f;
            }
            const int at = t.r * R + row;
            const int64_t o = (int64_t)(t.s.t0 + at / p.a.G) * p.a.heads * p.a.G + t.h * p.a.G + at % p.a.G;
            store_result(p.O + o * p.D + d, O, l > 0.0f ? 1.0f / l : 0.0f);
            if (p.lse && d == 0) p.lse[o] = result_lse(m, l);
        }
        return;
    }
}

template <int DP, int QT>
hipError_t launch(const AttnArgs& p, hipStream_t st) {
    constexpr int NW = DP * QT <= 128 ? 8 : 4;
    constexpr int bytes = NW * 16 * QT * (DP + 4 + 2) * (int)sizeof(float);
    static std::atomic<int> set[kMaxDevices];
    if (p.a.workers != p.a.groups * NW) return hipErrorInvalidConfiguration;
    const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(&attn_wave_kernel<DP, QT, NW>), bytes, set);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((attn_wave_kernel<DP, QT, NW>), dim3((unsigned)attn_grid(p.a)), dim3(NW * kWave), bytes, st, p);
    return hipGetLastError();
}

template <int DP>
hipError_t launch_rows(const AttnArgs& p, hipStream_t st) {
    return p.a.rows == 16 ? launch<DP, 1>(p, st) : launch<DP, 2>(p, st);
}

}  // namespace

hipError_t launch_attn_wave(const AttnArgs& p, hipStream_t st) {
    return p.D <= 64 ? launch_rows<64>(p, st) : p.D <= 128 ? launch_rows<128>(p, st) : launch_rows<256>(p, st);
}

}  // namespace sq
