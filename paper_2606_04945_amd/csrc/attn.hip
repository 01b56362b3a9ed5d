// Attention over the paged 8-bit cache.
//
// out = sum_j w_j v_j with w = softmax(scale q . k_j) over the visible keys, one
// pass: running maximum m, sum l and accumulator O of each row; a step of 64 keys
// raises m to m', multiplies l and O by 2^(m - m') and adds the step's terms
// (logits are kept times log2 e).  Codes go to the fp16 matrix cores as they are,
// every int8 being an fp16; a page's key scale multiplies its logits and its value
// scale the softmax weights, both in fp32.  The weights are then rounded to fp16
// relative to the largest value scale seen so far (kept like the maximum), so that
// no weight leaves fp16's normal range because a scale is small.
//
// Both products are formed transposed, S^T = K Q^T and O^T = V^T P^T: the
// accumulator layout of S^T (a lane has one query's keys) is the operand layout
// of P^T if the keys of a step are dealt to matrix rows so that lane group g's
// accumulators hold keys 16 g .. 16 g + 15, and softmax weights never leave their
// lane.  Keys are row operands as stored ([token][D]), and so are the transposed
// values ([D][token]): 16 contiguous bytes a lane.
#include "attn_plan.hpp"
#include "tile_common.hpp"

namespace sq {
namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNone = -__builtin_inff();

struct AttnArgs {
    AttnShape a;
    const uint16_t* Q;
    int64_t q_token, q_head;
    const int8_t *k, *v;
    const float *k_scale, *v_scale;
    int pages, page, shift, D;      // page = 1 << shift
    const int32_t *cu, *lens, *table;
    int max_pages;
    float scale;                    // times log2 e
    uint16_t* O;
    float* lse;
    float* ws;
};

__device__ __forceinline__ AttnSeq load_attn_seq(const AttnArgs& p, int b) {
    return attn_seq(p.a, p.cu[b], p.cu[b + 1], p.lens[b]);
}

__device__ __forceinline__ int64_t wave_scan(int64_t v, int lane) {
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const int64_t up = __shfl_up(v, o, kWave);
        if (lane >= o) v += up;
    }
    return v;
}

// All sequences' weights, and those before sequence b (b <= B), by one wave.
__device__ int64_t total_weight(const AttnArgs& p, int lane) {
    int64_t sum = 0;
    for (int b = lane; b < p.a.B; b += kWave) sum += load_attn_seq(p, b).weight;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, kWave);
    return sum * p.a.heads;
}

__device__ int64_t weight_before(const AttnArgs& p, int b, int lane) {
    int64_t sum = 0;
    for (int i = lane; i < b; i += kWave) sum += load_attn_seq(p, i).weight;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, kWave);
    return sum * p.a.heads;
}

// The sequence that weight position x falls in, and the weight before it.
__device__ int find_weight(const AttnArgs& p, int64_t x, int lane, int64_t& before) {
    int64_t done = 0;
    for (int b0 = 0; b0 < p.a.B; b0 += kWave) {
        const int b = b0 + lane;
        const int64_t w = b < p.a.B ? load_attn_seq(p, b).weight * p.a.heads : 0;
        const int64_t upto = done + wave_scan(w, lane);
        const uint64_t past = __ballot(upto > x);
        if (past) {
            const int i = __builtin_ctzll(past);
            before = __shfl(upto - w, i, kWave);
            return b0 + i;
        }
        done = __shfl(upto, kWave - 1, kWave);
    }
    before = done;
    return p.a.B;
}

// 8 int8 codes as 8 halves, exactly: with the sign bit flipped a code is a byte
// u = code + 128, the half 0x6400 | u is 1024 + u, and 1152 comes off.
__device__ __forceinline__ h8 to_halves(uint32_t w0, uint32_t w1) {
    const h2 bias = {(_Float16)1152.0f, (_Float16)1152.0f};
    const uint32_t u0 = w0 ^ 0x80808080u, u1 = w1 ^ 0x80808080u;
    const uint32_t x[4] = {__builtin_amdgcn_perm(0x64646464u, u0, 0x04010400u),
                           __builtin_amdgcn_perm(0x64646464u, u0, 0x04030402u),
                           __builtin_amdgcn_perm(0x64646464u, u1, 0x04010400u),
                           __builtin_amdgcn_perm(0x64646464u, u1, 0x04030402u)};
    h8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const h2 t = __builtin_bit_cast(h2, x[i]) - bias;
        r[2 * i] = t[0];
        r[2 * i + 1] = t[1];
    }
    return r;
}

// over the four 16-lane groups of a wave
__device__ __forceinline__ float groups_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16, kWave));
    return fmaxf(x, __shfl_xor(x, 32, kWave));
}
__device__ __forceinline__ float groups_sum(float x) {
    x += __shfl_xor(x, 16, kWave);
    return x + __shfl_xor(x, 32, kWave);
}

// One wave is one worker: 16 rows a tile, every load straight to registers, no
// barrier.  DP: head size rounded up to 64, 128 or 256.
template <int DP>
__global__ __launch_bounds__(256) void attn_wave_kernel(AttnArgs p) {
    constexpr int P = DP / 64, DT = DP / 16;
    const int lane = threadIdx.x % kWave, c = lane % 16, g = lane / 16;
    const int worker = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * (blockDim.x / kWave) + threadIdx.x / kWave));
    if (worker >= p.a.workers) return;
    const int G = p.a.G, D = p.D;
    const int64_t total = total_weight(p, lane);
    int64_t at = attn_start(total, p.a.workers, worker);
    const int64_t end = attn_start(total, p.a.workers, worker + 1);
    if (at >= end) return;
    int64_t before;
    int b = find_weight(p, at, lane, before);
    while (at < end && b < p.a.B) {
        const AttnSeq q = load_attn_seq(p, b);
        if (q.weight == 0) {
            ++b;
            continue;
        }
        const int h = (int)((at - before) / q.weight);
        int r = attn_find_tile(q, at - before - h * q.weight);
        for (; r < q.tiles && at < end; ++r) {
            const int64_t weight = q.base + q.slope * r;
            const int64_t from = before + h * q.weight + attn_before(q, r);
            const int64_t x0 = at - from, x1 = min(end - from, weight);
            at = from + x1;
            const AttnSteps steps = attn_steps(p.a, q.s, r);
            const int k0 = attn_cut(x0, weight, steps.count), k1 = attn_cut(x1, weight, steps.count);
            const bool whole = k1 - k0 == steps.count && (steps.count > 0 || x0 == 0);
            if (k0 == k1 && !whole) continue;

            // this lane's row (column c of the transposed products)
            const int64_t row = (int64_t)r * 16 + c, rows = (int64_t)q.s.n * G;
            const bool in = row < rows;
            const int i = (int)((in ? row : rows - 1) / G), qh = h * G + (int)((in ? row : rows - 1) % G);
            const int t = q.s.t0 + i, pos = q.s.off + i;
            const int lo = attn_lo(p.a, pos), hi = attn_hi(p.a, q.s, pos);
            const uint16_t* qp = p.Q + t * p.q_token + qh * p.q_head;
            h8 Qf[2 * P];
#pragma unroll
            for (int s = 0; s < 2 * P; ++s) {
                const int d = 64 * (s / 2) + 16 * g + 8 * (s % 2);
                Qf[s] = d < D ? *reinterpret_cast<const h8*>(qp + d) : h8{};
            }
            f4 O[DT];
#pragma unroll
            for (int d = 0; d < DT; ++d) O[d] = f4{0, 0, 0, 0};
            float m = kNone, l = 0.0f, vref = 0.0f;
            const int32_t* table = p.table + (int64_t)b * p.max_pages;
            for (int kt = steps.first + k0; kt < steps.first + k1; ++kt) {
                // pages of this lane's key row (group c / 4) and of its accumulators' keys (group g)
                const int key0 = kt * kAttnStep;
                const int ka = key0 + 16 * (c / 4), va = key0 + 16 * g;
                const int kp = ka < q.s.len ? table[ka >> p.shift] : -1;
                const int vp = va < q.s.len ? table[va >> p.shift] : -1;
                const bool kin = (uint32_t)kp < (uint32_t)p.pages, vin = (uint32_t)vp < (uint32_t)p.pages;
                const int64_t kph = kin ? (int64_t)kp * p.a.heads + h : h, vph = vin ? (int64_t)vp * p.a.heads + h : h;
                const int8_t* kr = p.k + (kph * p.page + (ka & (p.page - 1)) + c % 4) * D + 16 * g;
                const int8_t* vr = p.v + vph * p.page * D + (va & (p.page - 1));
                v4i kw[4][P], vw[DT];
#pragma unroll
                for (int s = 0; s < 4; ++s)
#pragma unroll
                    for (int z = 0; z < P; ++z)
                        kw[s][z] = 64 * z + 16 * g < D ? *reinterpret_cast<const v4i*>(kr + 4 * s * D + 64 * z)
                                                       : v4i{0, 0, 0, 0};
                const float ks = p.k_scale[vph] * p.scale, vs0 = p.v_scale[vph];
#pragma unroll
                for (int d = 0; d < DT; ++d)
                    vw[d] = *reinterpret_cast<const v4i*>(vr + min(16 * d + c, D - 1) * p.page);
                f4 S[4];
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    S[s] = f4{0, 0, 0, 0};
#pragma unroll
                    for (int z = 0; z < P; ++z)
#pragma unroll
                        for (int y = 0; y < 2; ++y)
                            S[s] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                                to_halves((uint32_t)kw[s][z][2 * y], (uint32_t)kw[s][z][2 * y + 1]), Qf[2 * z + y], S[s],
                                0, 0, 0);
                }
                float mx = kNone;
                if (__all(vin && key0 >= lo && key0 + kAttnStep <= hi)) {
#pragma unroll
                    for (int s = 0; s < 4; ++s)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            S[s][e] *= ks;
                            mx = fmaxf(mx, S[s][e]);
                        }
                } else {
#pragma unroll
                    for (int s = 0; s < 4; ++s)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int key = va + 4 * s + e;
                            S[s][e] = vin && key >= lo && key < hi ? S[s][e] * ks : kNone;
                            mx = fmaxf(mx, S[s][e]);
                        }
                }
                const float mn = fmaxf(m, groups_max(mx));
                const float ms = mn == kNone ? 0.0f : mn;       // a row that has seen nothing yet: all terms 0
                const float vs = vin && va < hi && va + 16 > lo ? vs0 : 0.0f;   // not of keys no term takes
                const float vn = fmaxf(vref, groups_max(vs));
                const float vi = vn > 1e-37f ? 1.0f / vn : 0.0f;
                const float fade = __builtin_amdgcn_exp2f(m - ms);
                const float turn = fade * (vref * vi), part = vs * vi;
                m = mn;
                vref = vn;
                float sum = 0.0f;
                h8 Pf[2];
#pragma unroll
                for (int s = 0; s < 4; ++s)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float w = __builtin_amdgcn_exp2f(S[s][e] - ms);
                        sum += w;
                        Pf[s / 2][4 * (s % 2) + e] = (_Float16)(w * part);
                    }
                l = l * fade + sum;
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    O[d] *= turn;
                    O[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(to_halves((uint32_t)vw[d][0], (uint32_t)vw[d][1]), Pf[0],
                                                                 O[d], 0, 0, 0);
                    O[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(to_halves((uint32_t)vw[d][2], (uint32_t)vw[d][3]), Pf[1],
                                                                 O[d], 0, 0, 0);
                }
            }
            l = groups_sum(l);
            if (whole) {
                if (in) {
                    const float inv = l > 0.0f ? vref / l : 0.0f;
                    uint16_t* op = p.O + ((int64_t)t * p.a.heads * G + qh) * D + 4 * g;
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        if (16 * d >= D) break;
                        uint2 w;
                        w.x = (uint32_t)f2h(O[d][0] * inv) | ((uint32_t)f2h(O[d][1] * inv) << 16);
                        w.y = (uint32_t)f2h(O[d][2] * inv) | ((uint32_t)f2h(O[d][3] * inv) << 16);
                        *reinterpret_cast<uint2*>(op + 16 * d) = w;
                    }
                    if (p.lse && g == 0)
                        p.lse[(int64_t)t * p.a.heads * G + qh] = l > 0.0f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : kNone;
                }
            } else {
                float* ws = p.ws + attn_place(worker, x0 > 0) * (int64_t)(16 * (D + 2));
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    if (16 * d >= D) break;
                    *reinterpret_cast<f4*>(ws + c * D + 16 * d + 4 * g) = O[d] * vref;
                }
                if (g == 0) ws[16 * D + c] = m, ws[16 * D + 16 + c] = l;
            }
        }
        if (r == q.tiles && at - before >= q.weight * p.a.heads) {
            before += q.weight * p.a.heads;
            ++b;
        }
    }
}

// Joins the partial results of one tile: out = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i,
// in the workers' order, so the result does not depend on which ended first.
constexpr int kJoinThreads = 256;
__global__ __launch_bounds__(kJoinThreads) void attn_join_kernel(AttnArgs p) {
    __shared__ int places[kJoinThreads];
    __shared__ int counts[kJoinThreads / kWave];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int R = p.a.rows, D = p.D, G = p.a.G;
    // the sequence whose list of tiles holds this workgroup's
    int lo = 0, hi = p.a.B - 1;
    const int64_t item = blockIdx.x / p.a.heads;
    const int h = blockIdx.x % p.a.heads;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        const int cm = min(max(p.cu[mid], 0), p.a.T);
        if (list_start(cm, mid, G, R, 1) <= item) lo = mid; else hi = mid - 1;
    }
    const int b = lo;
    const AttnSeq q = load_attn_seq(p, b);
    const int64_t r64 = item - list_start(q.s.t0, b, G, R, 1);
    if (r64 < 0 || r64 >= q.tiles) return;
    const int r = (int)r64;
    const AttnSteps steps = attn_steps(p.a, q.s, r);
    if (steps.count <= 1) return;                 // never split
    const int64_t total = total_weight(p, lane);
    const int64_t from = weight_before(p, b, lane) + h * q.weight + attn_before(q, r);
    const int64_t weight = q.base + q.slope * r;
    const int w0 = attn_worker(total, p.a.workers, from), w1 = attn_worker(total, p.a.workers, from + weight - 1);
    if (w0 == w1) return;
    const int64_t size = attn_place_floats(R, D);
    const int rows = (int)min((int64_t)R, (int64_t)q.s.n * G - (int64_t)r * R);
    const int vecs = D / 4;
    // each thread: four channels of some rows; partial results in batches of kJoinThreads
    for (int e0 = 0; e0 < rows * vecs; e0 += kJoinThreads) {
        const int e = e0 + tid;
        const bool mine = e < rows * vecs;
        const int row = mine ? e / vecs : 0, d = mine ? e % vecs * 4 : 0;
        float m = kNone, l = 0.0f;
        f4 O{0, 0, 0, 0};
        for (int wb = w0; wb <= w1; wb += kJoinThreads) {
            const int w = wb + tid;
            int place = -1;
            bool alone = false;
            if (w <= w1) {
                const int64_t x0 = attn_start(total, p.a.workers, w) - from;
                const int64_t x1 = min(attn_start(total, p.a.workers, w + 1) - from, weight);
                const int k0 = attn_cut(x0, weight, steps.count), k1 = attn_cut(x1, weight, steps.count);
                alone = k1 - k0 == steps.count;
                if (k1 > k0) place = attn_place(w, x0 > 0);
            }
            if (__syncthreads_or(alone)) return;          // one worker had every step and wrote the rows
            const uint64_t some = __ballot(place >= 0);
            if (lane == 0) counts[wave] = __popcll(some);
            __syncthreads();
            int base = 0, n = 0;
#pragma unroll
            for (int v = 0; v < kJoinThreads / kWave; ++v) {
                if (v < wave) base += counts[v];
                n += counts[v];
            }
            if (place >= 0) places[base + __popcll(some & ((1ull << lane) - 1))] = place;
            __syncthreads();
            for (int j = 0; j < n; ++j) {
                const float* ws = p.ws + places[j] * size;
                const float mj = ws[R * D + row], lj = ws[R * D + R + row];
                const f4 Oj = *reinterpret_cast<const f4*>(ws + row * D + d);
                const float mn = fmaxf(m, mj), ms = mn == kNone ? 0.0f : mn;
                const float f = __builtin_amdgcn_exp2f(m - ms), fj = __builtin_amdgcn_exp2f(mj - ms);
                O = O * f + Oj * fj;
                l = l * f + lj * fj;
                m = mn;
            }
            __syncthreads();
        }
        if (!mine) continue;
        const int64_t rr = (int64_t)r * R + row;
        const int64_t o = (int64_t)(q.s.t0 + (int)(rr / G)) * p.a.heads * G + h * G + (int)(rr % G);
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        uint2 w;
        w.x = (uint32_t)f2h(O[0] * inv) | ((uint32_t)f2h(O[1] * inv) << 16);
        w.y = (uint32_t)f2h(O[2] * inv) | ((uint32_t)f2h(O[3] * inv) << 16);
        *reinterpret_cast<uint2*>(p.O + o * D + d) = w;
        if (p.lse && d == 0) p.lse[o] = l > 0.0f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : kNone;
    }
}

AttnShape wave_shape(int T, int B, int Hq, int heads, int max_len, bool causal, int window) {
    AttnShape a{T, B, heads, Hq / heads, max_len, causal, window, 16, 0};
    a.workers = attn_workers(a, kAttnWaves);
    return a;
}

bool never_split(const AttnShape& a) { return a.max_len <= kAttnStep; }

}  // namespace

size_t attn_workspace_bytes(int T, int B, int Hq, int heads, int D, int max_len) {
    const AttnShape a = wave_shape(T, B, Hq, heads, max_len, true, 0);
    return never_split(a) ? 0 : (size_t)a.workers * 2 * attn_place_floats(a.rows, D) * sizeof(float);
}

hipError_t launch_attn(const uint16_t* Q, int64_t q_token, int64_t q_head, const int8_t* k, const int8_t* v,
                       const float* k_scale, const float* v_scale, int pages, int page, int heads, int D,
                       const int32_t* cu, const int32_t* lens, const int32_t* table, int T, int B, int max_pages, int Hq,
                       bool causal, int window, float scale, uint16_t* O, float* lse, void* ws, hipStream_t st) {
    const AttnShape a = wave_shape(T, B, Hq, heads, max_pages * page, causal, window);
    const AttnArgs p{a, Q, q_token, q_head, k, v, k_scale, v_scale, pages, page, __builtin_ctz((unsigned)page), D,
                     cu, lens, table, max_pages, scale * kLog2e, O, lse, static_cast<float*>(ws)};
    const dim3 grid((unsigned)((a.workers + 3) / 4));
    if (D <= 64)
        hipLaunchKernelGGL(attn_wave_kernel<64>, grid, dim3(256), 0, st, p);
    else if (D <= 128)
        hipLaunchKernelGGL(attn_wave_kernel<128>, grid, dim3(256), 0, st, p);
    else
        hipLaunchKernelGGL(attn_wave_kernel<256>, grid, dim3(256), 0, st, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || never_split(a)) return e;
    hipLaunchKernelGGL(attn_join_kernel, dim3((unsigned)attn_tile_slots(a)), dim3(kJoinThreads), 0, st, p);
    return hipGetLastError();
}

}  // namespace sq
