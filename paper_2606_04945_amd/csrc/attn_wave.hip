// Attention over the paged 8-bit cache for few rows: every load goes straight to
// registers and no wave waits for another inside the loop over keys.
//
// The matrix instruction is 16 x 16 x 32.  Matrix row c of key tile s is key
// 16 (c / 4) + 4 s + c % 4 of the step, so lane group g's four accumulators hold keys
// 16 g .. 16 g + 15, and it reads its values as 16 contiguous bytes a channel; keys
// are read as 16 contiguous channels.  A lane group's keys share a page, and with it
// one pair of scales.
//
// Bound by reading the codes where there are many of them (2 x 131072 keys of 8 heads of
// 128: 97 us, 4.9 TB/s; 32 next tokens over 6000 keys on average 38 us, 5.2 TB/s, the
// joining apart); by the round trips of a step where there are few (one token of 32
// heads over 518 keys: 10.6 us in a series of calls); by the longest tile's steps where a
// batch is read tile by tile (8 blocks of 32 tokens of 32 heads over up to 2080 keys: 36 us,
// 3.1 TB/s).
#include "attn_common.hpp"

namespace sq {
namespace {

constexpr float kLargest = 14.0f;     // log2 of a row's largest weight

// over the four 16-lane groups of a wave
__device__ __forceinline__ float groups_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16, kWave));
    return fmaxf(x, __shfl_xor(x, 32, kWave));
}
__device__ __forceinline__ float groups_sum(float x) {
    x += __shfl_xor(x, 16, kWave);
    return x + __shfl_xor(x, 32, kWave);
}

// A load that the scheduler leaves in its place.  What enters a loop and what comes
// round it then have the same loads in flight in the same order, and the wait for one
// of them need not be a wait for all.
template <class T>
__device__ __forceinline__ T load_in_order(const void* p) {
    const T x = *static_cast<const T*>(p);
    __builtin_amdgcn_sched_barrier(0);
    return x;
}

// One wave's rows of a tile: 16 QT of them, and the pass over some of their steps.
// DP: head size rounded up to 64, 128 or 256.  WIDE: pages of 64 tokens and more.
template <int DP, int QT, bool WIDE>
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
                Q[y][z] = d < p.D ? load_query(q + d) : h8{};
            }
            m[y] = kUnseen, l[y] = 0.0f;
#pragma unroll
            for (int d = 0; d < DT; ++d) O[y][d] = f4{0, 0, 0, 0};
        }
    }

    // What a step reads, a lane's part.  Every load is issued on every step (addresses are
    // kept inside instead), so that waiting for some leaves the others in flight.
    struct Reads {
        bool in;                                  // this lane group's keys have a page
        v4i k[4][P], v[DT];
        float ks, vs;
    };

    // The pass over steps first, first + stride, ... below end.  64 page table entries are
    // held, one a lane, in the order in which the steps need them.
    struct Pages {
        const int32_t* table;
        int held, first, stride;                  // entries of the sequence; the steps
        int per, ids;                             // entries a step; this lane's page, -1: none
    };
    __device__ __forceinline__ void hold(const AttnArgs& p, Pages& q, int j, int lane) const {
        const int at = ((q.first + (j + lane / q.per) * q.stride) * kAttnStep >> p.shift) + lane % q.per;
        const int id = q.table[min(at, q.held - 1)];
        q.ids = at < q.held && (uint32_t)id < (uint32_t)p.pages ? id : -1;
    }
    __device__ __forceinline__ int64_t head_of(const AttnArgs& p, int pid, int h) const {
        return pid >= 0 ? (int64_t)pid * p.a.heads + h : (int64_t)h;
    }
    // Keys and scales, and values, of the pass's step j.  WIDE: one page a step, addresses
    // from scalar registers; otherwise a lane has the page of its key row (group c / 4 of the
    // step) and that of its lane group.  Past the channels the keys are others again, which
    // meet zero queries, and the values too, which are not stored.
    __device__ __forceinline__ void keys(const AttnArgs& p, const Pages& q, int h, int j, int c, int g,
                                         Reads& r) const {
        const int key0 = (q.first + j * q.stride) * kAttnStep, entry = j * q.per & (kWave - 1);
        int64_t ph;
        const int8_t* at;
        if (WIDE) {
            const int pid = __builtin_amdgcn_readlane(q.ids, entry);
            r.in = pid >= 0;
            ph = head_of(p, pid, h);
            at = p.k + (ph * p.page + (key0 & (p.page - 1))) * p.D;
        } else {
            const int kp = __shfl(q.ids, entry + (16 * (c / 4) >> p.shift), kWave);
            const int vp = __shfl(q.ids, entry + (16 * g >> p.shift), kWave);
            r.in = vp >= 0;
            ph = head_of(p, vp, h);
            at = p.k + (head_of(p, kp, h) * p.page + (16 * (c / 4) & (p.page - 1)) - 16 * (c / 4)) * p.D;
        }
        const int row = (16 * (c / 4) + c % 4) * p.D;
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int z = 0; z < P; ++z)
                r.k[e][z] = load_in_order<v4i>(at + 4 * e * p.D + (uint32_t)(row + min(64 * z + 16 * g, p.D - 16)));
        r.ks = load_in_order<float>(p.k_scale + ph);
        r.vs = load_in_order<float>(p.v_scale + ph);
    }
    __device__ __forceinline__ void values(const AttnArgs& p, const Pages& q, int h, int j, int c, int g,
                                           Reads& r) const {
        const int key0 = (q.first + j * q.stride) * kAttnStep, entry = j * q.per & (kWave - 1);
        const int8_t* at;
        if (WIDE) {
            at = p.v + head_of(p, __builtin_amdgcn_readlane(q.ids, entry), h) * p.page * p.D + (key0 & (p.page - 1));
        } else {
            const int vp = __shfl(q.ids, entry + (16 * g >> p.shift), kWave);
            at = p.v + head_of(p, vp, h) * p.page * p.D + (16 * g & (p.page - 1)) - 16 * g;
        }
#pragma unroll
        for (int d = 0; d < DT; ++d)
            r.v[d] = load_in_order<v4i>(at + min(16 * d, p.D - 16) * p.page + (uint32_t)(c * p.page + 16 * g));
    }

    // What the next step reads is requested as soon as the registers of this one's are
    // free: its keys before this step's softmax, its values after the second product.
    __device__ __forceinline__ void pass(const AttnArgs& p, const Seq& s, int b, int h, int first, int end, int stride,
                                         int lane) {
        const int c = lane % 16, g = lane / 16;
        if (first < end) {
            const int n = (end - first + stride - 1) / stride, per = WIDE ? 1 : kAttnStep >> p.shift;
            Pages q{p.table + (int64_t)b * p.max_pages, (s.len + p.page - 1) >> p.shift, first, stride, per, -1};
            Reads r;
            hold(p, q, 0, lane);
            keys(p, q, h, 0, c, g, r);
            values(p, q, h, 0, c, g, r);
#pragma unroll
            for (int y = 0; y < QT; ++y)
#pragma unroll
                for (int z = 0; z < 2 * P; ++z) Q[y][z] = flip_query(Q[y][z], p.flip);
            for (int j = 0; j + 1 < n; ++j) step<true>(p, q, h, j, lane, r);
            step<false>(p, q, h, n - 1, lane, r);
        }
#pragma unroll
        for (int y = 0; y < QT; ++y) {
            l[y] = groups_sum(l[y]);
            // no weight at all: products of -inf, where a query is infinite
            const bool none = first < end && l[y] == 0.0f && lo[y] < hi[y];
            if (__any(none)) {
                const float fault = groups_sum(query_fault(Q[y]));
                if (none) l[y] = fault;
            }
        }
    }

    template <bool MORE>
    __device__ __forceinline__ void step(const AttnArgs& p, Pages& q, int h, int j, int lane, Reads& r) {
        const int c = lane % 16, g = lane / 16;
        const int key0 = (q.first + j * q.stride) * kAttnStep, va = key0 + 16 * g;
        const BlockScale bs = block_scale(r.in, r.ks, r.vs, p.scale);
        f4 S[QT][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
            for (int y = 0; y < QT; ++y) S[y][e] = f4{0, 0, 0, 0};
#pragma unroll
            for (int z = 0; z < 2 * P; ++z) {
                const v4i w = r.k[e][z / 2];
                const h8 k = to_halves((uint32_t)w[2 * (z % 2)], (uint32_t)w[2 * (z % 2) + 1]);
#pragma unroll
                for (int y = 0; y < QT; ++y)
                    S[y][e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, Q[y][z], S[y][e], 0, 0, 0);
            }
        }
        if (MORE) {
            if (((j + 1) * q.per & (kWave - 1)) == 0) hold(p, q, j + 1, lane);
            keys(p, q, h, j + 1, c, g, r);
        }
        float top[QT], most = 0.0f, ks = bs.ks, lv = bs.lv;
#pragma unroll
        for (int y = 0; y < QT; ++y) {
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
            mx = groups_max(__builtin_fmaf(mx, ks, lv));
            top[y] = mx - kLargest;
            most = fmaxf(most, fabsf(mx));
        }
        if (__any(most > kFine)) {
#pragma unroll
            for (int y = 0; y < QT; ++y) {
                float mx = kNone;
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        S[y][e][i] = __builtin_fmaf(S[y][e][i], ks, lv);
                        mx = fmaxf(mx, S[y][e][i]);
                    }
                mx = groups_max(mx);
                if (fabsf(mx) > kFine) top[y] = mx;
            }
            ks = 1.0f, lv = 0.0f;
        }
        h8 W[QT][2];
#pragma unroll
        for (int y = 0; y < QT; ++y) {
            const float mx = fmaxf(m[y], top[y]);
            const float fade = __builtin_amdgcn_exp2f(m[y] - mx), off = lv - mx;
            m[y] = mx;
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    const f2 w = {__builtin_amdgcn_exp2f(__builtin_fmaf(S[y][e][i], ks, off)),
                                  __builtin_amdgcn_exp2f(__builtin_fmaf(S[y][e][i + 1], ks, off))};
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
                const h8 v = to_halves((uint32_t)r.v[d][2 * u], (uint32_t)r.v[d][2 * u + 1]);
#pragma unroll
                for (int y = 0; y < QT; ++y)
                    O[y][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, W[y][u], O[y][d], 0, 0, 0);
            }
        if (MORE) values(p, q, h, j + 1, c, g, r);
    }

    __device__ __forceinline__ void store(const AttnArgs& p, int g) const {
#pragma unroll
        for (int y = 0; y < QT; ++y) {
            if (!in[y]) continue;
            const float inv = inverse(m[y], l[y]);
            const int64_t o = (int64_t)t[y] * p.a.heads * p.a.G + qh[y];
#pragma unroll
            for (int d = 0; d < DT; ++d)
                if (16 * d < p.D) store_result(p.O + o * p.D + 16 * d + 4 * g, O[y][d], inv);
            if (p.lse && g == 0) store_global(p.lse + o, result_lse(m[y], l[y]));
        }
    }

    // `any` false: this worker's place of the tile holds nothing to join
    __device__ __forceinline__ void store_partial(const AttnArgs& p, float* ws, bool any, int c, int g) const {
        constexpr int R = 16 * QT;
#pragma unroll
        for (int y = 0; y < QT; ++y) {
            if (!in[y]) continue;
            const int row = 16 * y + c;
            if (any) {
#pragma unroll
                for (int d = 0; d < DT; ++d)
                    if (16 * d < p.D) store_global(ws + row * p.D + 16 * d + 4 * g, O[y][d]);
            }
            if (g == 0) {
                store_global(ws + R * p.D + row, any ? m[y] : kNone);
                store_global(ws + R * p.D + R + row, l[y]);
            }
        }
    }
};

// Direct: a workgroup is a tile, whose steps go round its waves, and their results
// meet in LDS.  Otherwise every wave is a worker of the shared work.
template <int DP, int QT, int NW, bool WIDE>
__global__ __launch_bounds__(NW* kWave) void attn_wave_kernel(AttnArgs p) {
    extern __shared__ __attribute__((aligned(16))) float lds[];
    constexpr int R = 16 * QT, LD = DP + 4;            // rows, padded row of floats
    __builtin_assume(p.a.rows == R);
    float* ml = lds + NW * R * LD;                     // [wave][row] m, then l
    const int lane = threadIdx.x % kWave, c = lane % 16, g = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const Group first = load_group(p, 0, lane);
    const Survey all = survey(p, first, lane);
    Share sh{};
    Tile t{};
    int stride = 1, count = 0;
    const int worker = worker_of(p, all, wave, NW);
    if (!attn_always_direct(p.a) && blockIdx.x == 0 && threadIdx.x == 0) store_global(p.shared, (int)!all.direct);
    if (all.direct) {
        const int item = (int)blockIdx.x / p.a.heads;
        const Listed at = find_listed(p, item, first, lane);
        const int64_t r64 = item - list_start(at.q.s.t0, at.b, p.a.G, R, 1);
        if (r64 < 0 || r64 >= at.q.tiles) return;
        const AttnSteps steps = attn_steps(p.a, at.q.s, (int)r64);
        count = steps.count;
        stride = NW;
        t = {at.q.s, at.b, (int)blockIdx.x % p.a.heads, (int)r64,
             {0, steps.first + wave, steps.first + steps.count, false, false, false}};
    } else {
        if ((int)blockIdx.x >= p.a.groups) return;
        if (lane == 0) store_global(p.lasts + worker, -1);
        sh = find_share(p, all.total, first, worker, lane);
    }
    for (;;) {
        if (!all.direct && !next_tile<true>(p, first, sh, worker, t)) return;
        WaveRows<DP, QT, WIDE> w;
        w.begin(p, t.s, t.h, t.r, c, g);
        w.pass(p, t.s, t.b, t.h, t.part.k0, t.part.k1, stride, lane);
        if (!all.direct) {
            if (t.part.whole) w.store(p, g);
            if (t.part.begins_inside || t.part.ends_inside)
                w.store_partial(p, p.places + attn_place(worker, t.part.begins_inside) * attn_place_floats(R, p.D),
                                t.part.k0 < t.part.k1 && !t.part.whole, c, g);
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
            store_result(p.O + o * p.D + d, O, inverse(m, l));
            if (p.lse && d == 0) store_global(p.lse + o, result_lse(m, l));
        }
        return;
    }
}

template <int DP, int QT, bool WIDE>
hipError_t launch_pages(const AttnArgs& p, hipStream_t st) {
    constexpr int NW = DP * QT <= 128 ? 8 : 4;
    constexpr int bytes = NW * 16 * QT * (DP + 4 + 2) * (int)sizeof(float);
    static std::atomic<int> set[kMaxDevices];
    if (p.a.workers != p.a.groups * NW) return hipErrorInvalidConfiguration;
    const auto kernel = &attn_wave_kernel<DP, QT, NW, WIDE>;
    const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), bytes, set);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)attn_grid(p.a)), dim3(NW * kWave), bytes, st, p);
    return hipGetLastError();
}

template <int DP, int QT>
hipError_t launch(const AttnArgs& p, hipStream_t st) {
    return p.page >= kAttnStep ? launch_pages<DP, QT, true>(p, st) : launch_pages<DP, QT, false>(p, st);
}

}  // namespace

hipError_t launch_attn_wave(const AttnArgs& p, hipStream_t st) {
    const bool two = p.a.rows == 32;
    if (p.D <= 64) return two ? launch<64, 2>(p, st) : launch<64, 1>(p, st);
    if (p.D <= 128) return two ? launch<128, 2>(p, st) : launch<128, 1>(p, st);
    return two ? hipErrorInvalidConfiguration : launch<256, 1>(p, st);
}

}  // namespace sq
