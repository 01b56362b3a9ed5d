// Rotary positions and the paged 8-bit key / value cache: rotation, append, and
// reading pages back.
//
// A page holds `page` tokens of every key head; its keys are [head][token][D] and
// its values [head][D][token], so that the attention kernels read both as matrix
// operands without a transpose.  Codes are int8 with one fp32 scale for each page
// and head, s = absmax / 127.
#include "kv_plan.hpp"
#include "rope.hpp"

namespace sq {
namespace {

constexpr int kThreads = 256;

// ---- frequencies ---------------------------------------------------------------------------------------------

// f_j = base^(-2j / rot) radians per position, stretched for contexts `factor`
// times the original: linear f / factor; ntk: base times factor^(rot / (rot - 2)),
// which leaves pair 0 and stretches the last by factor; yarn: pairs that turn
// beta_fast times or more over the original context stay, those that turn beta_slow
// times or fewer are stretched, linear in the turns between.
__global__ void rope_frequencies_kernel(int rot, double base, int scaling, double factor, double original,
                                        double beta_fast, double beta_slow, double* __restrict__ freq) {
    const int j = blockIdx.x * kThreads + threadIdx.x;
    if (j >= rot / 2) return;
    if (scaling == 2 && rot > 2) base *= pow(factor, (double)rot / (rot - 2));
    double f = pow(base, -2.0 * j / rot);
    if (scaling == 1) f /= factor;
    if (scaling == 3) {
        const double turns = original * f / 6.283185307179586477;
        double keep = (turns - beta_slow) / (beta_fast - beta_slow);
        keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
        f = f * keep + f / factor * (1 - keep);
    }
    freq[j] = f;
}

// ---- rotation ------------------------------------------------------------------------------------------------

struct RopeArgs {
    const uint16_t* X;
    int64_t x_token, x_head;
    uint16_t* Y;
    int64_t y_token, y_head;
    const double* freq;
    int T, H, D, rot, layout;
    bool transpose;
    float amp;
};

// One unit of `heads` heads of one token: the unit's angles are formed once for
// all of them (an fp64 product and a sine and cosine each).
template <int VEC>
__device__ __forceinline__ void rotate_unit(const RopeArgs& a, int t, int pos, int h0, int heads, int u) {
    const RopeUnit r = rope_unit<VEC>(u, a.rot, a.layout);
    float c[VEC], s[VEC];
    if (r.pair >= 0) {
#pragma unroll
        for (int q = 0; q < VEC; ++q) rope_angle(pos, a.freq[r.pair + q], a.amp, a.transpose, c[q], s[q]);
    }
    const uint16_t* x = a.X + t * a.x_token + h0 * a.x_head;
    uint16_t* y = a.Y + t * a.y_token + h0 * a.y_head;
    for (int h = 0; h < heads; ++h, x += a.x_head, y += a.y_head) {
        float p[VEC], q[VEC];
        load_run<VEC>(x + r.a, p);
        load_run<VEC>(x + r.b, q);
        if (r.pair >= 0) rope_turn<VEC>(p, q, c, s, a.layout);
        store_run<VEC>(y + r.a, p);
        store_run<VEC>(y + r.b, q);
    }
}

// One thread: one unit of `per` heads of one token.
template <int VEC>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a, const int32_t* __restrict__ pos, int per) {
    const int units = a.D / (2 * VEC), groups = (a.H + per - 1) / per;
    const int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int u = (int)(e % units);
    const int64_t tg = e / units;
    const int g = (int)(tg % groups);
    if (tg / groups >= a.T) return;
    const int t = (int)(tg / groups);
    const int h0 = g * per;
    rotate_unit<VEC>(a, t, pos ? pos[t] : t, h0, min(per, a.H - h0), u);
}

// ---- append --------------------------------------------------------------------------------------------------

struct AppendArgs {
    int8_t *k, *v;
    float *k_scale, *v_scale;
    int pages, page, heads, D;
    const uint16_t *K, *V;
    int64_t k_token, k_head, v_token, v_head;
    const int32_t *cu, *lens, *table, *pos;
    int T, B, max_pages;
    const double* freq;
    int rot, layout;
    float amp;
};

__device__ __forceinline__ Seq load_seq(const int32_t* cu, const int32_t* lens, int b, int T, int max_len) {
    return make_seq(cu[b], cu[b + 1], lens[b], T, max_len);
}

// The last b with list_start(b) <= i, for non-decreasing starts (clamped rows).
__device__ __forceinline__ int find_seq(const int32_t* cu, int B, int T, int64_t i, int per, int size, int extra) {
    int lo = 0, hi = B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        const int c = min(max(cu[mid], 0), T);
        if (list_start(c, mid, per, size, extra) <= i) lo = mid; else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ float block_max(float x, float* red) {
    x = wave_max(x);
    __syncthreads();
    if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = x;
    __syncthreads();
    x = red[0];
#pragma unroll
    for (int w = 1; w < kThreads / kWave; ++w) x = fmaxf(x, red[w]);
    return x;
}

// x 127 codes against scale s, y = 1 / s; s = 0: zero codes
__device__ __forceinline__ void codes16(const float (&x)[16], float s, float y, uint32_t (&w)[4]) {
    int c[16];
    quant_codes8<127>(x, s, y, c);
    quant_codes8<127>(x + 8, s, y, c + 8);
#pragma unroll
    for (int q = 0; q < 4; ++q)
        w[q] = s > 0.0f ? (uint32_t)(c[4 * q] & 255) | ((uint32_t)(c[4 * q + 1] & 255) << 8) |
                              ((uint32_t)(c[4 * q + 2] & 255) << 16) | ((uint32_t)(c[4 * q + 3] & 255) << 24)
                        : 0u;
}

__device__ __forceinline__ uint32_t rescale4(uint32_t w, float ratio) {
    uint32_t r = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int c = (int)__builtin_rintf((float)(int8_t)(w >> (8 * q)) * ratio);
        r |= (uint32_t)(c & 255) << (8 * q);
    }
    return r;
}

// One workgroup: the new tokens of one page for one key head.  Pass 1 stages the
// rotated keys (fp32) in LDS and takes their absmax, the codes follow; then the
// same for the values, transposed on the way out.  The workgroup owns the page's
// codes of its head, so a growing scale requantises the older codes in place:
// code' = rint(code s / s').
template <int VEC>
__device__ void append_block(const AppendArgs& a, int64_t item, int h, float* lds, float* red) {
    const int b = find_seq(a.cu, a.B, a.T, item, 1, a.page, 2);
    const Seq s = load_seq(a.cu, a.lens, b, a.T, a.max_pages * a.page);
    const int64_t j = item - list_start(s.t0, b, 1, a.page, 2);
    if (j < 0 || j >= touched_count(s, a.page)) return;
    const int blk = touched_first(s, a.page) + (int)j;
    const int pid = a.table[(int64_t)b * a.max_pages + blk];
    if ((uint32_t)pid >= (uint32_t)a.pages) return;
    const int p0 = max(s.off, blk * a.page), p1 = min(s.len, (blk + 1) * a.page);   // positions written
    const int s0 = p0 - blk * a.page, s1 = p1 - blk * a.page, n = s1 - s0;
    const int row0 = s.t0 + p0 - s.off;
    const int D = a.D, tid = threadIdx.x;
    const int64_t ph = (int64_t)pid * a.heads + h;
    int8_t* kc = a.k + ph * a.page * D;
    int8_t* vc = a.v + ph * a.page * D;
    const float ks0 = s0 ? a.k_scale[ph] : 0.0f, vs0 = s0 ? a.v_scale[ph] : 0.0f;

    const int units = D / (2 * VEC);
    float m = 0.0f;
    for (int e = tid; e < n * units; e += kThreads) {
        const int i = e / units;
        const int t = row0 + i;
        const uint16_t* x = a.K + t * a.k_token + h * a.k_head;
        float p[VEC], q[VEC];
        const RopeUnit r = a.freq ? rope_unit<VEC>(e % units, a.rot, a.layout) : rope_unit<VEC>(e % units, 0, 0);
        load_run<VEC>(x + r.a, p);
        load_run<VEC>(x + r.b, q);
        if (r.pair >= 0) {
            const int pos = a.pos ? a.pos[t] : p0 + i;
            float c[VEC], sn[VEC];
#pragma unroll
            for (int z = 0; z < VEC; ++z) rope_angle(pos, a.freq[r.pair + z], a.amp, false, c[z], sn[z]);
            rope_turn<VEC>(p, q, c, sn, a.layout);
        }
#pragma unroll
        for (int z = 0; z < VEC; ++z) {
            m = fmaxf(m, fmaxf(fabsf(p[z]), fabsf(q[z])));
            lds[i * D + r.a + z] = p[z];
            lds[i * D + r.b + z] = q[z];
        }
    }
    m = block_max(m, red);
    float sc = fmaxf(ks0, m / 127.0f);
    float y = 1.0f / sc;
    if (s0 && sc > ks0) {
        const float ratio = ks0 / sc;
        for (int e = tid; e < s0 * D / 4; e += kThreads) {
            uint32_t* w = reinterpret_cast<uint32_t*>(kc) + e;
            *w = rescale4(*w, ratio);
        }
    }
    for (int e = tid; e < n * D / 16; e += kThreads) {
        float x[16];
#pragma unroll
        for (int z = 0; z < 16; ++z) x[z] = lds[e * 16 + z];
        uint32_t w[4];
        codes16(x, sc, y, w);
        *reinterpret_cast<v4i*>(kc + s0 * D + e * 16) = v4i{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
    }
    if (tid == 0) a.k_scale[ph] = sc;

    __syncthreads();
    m = 0.0f;
    for (int e = tid; e < n * (D / 8); e += kThreads) {
        const int i = e / (D / 8), d = e % (D / 8) * 8;
        float x[8];
        load_run<8>(a.V + (row0 + i) * a.v_token + h * a.v_head + d, x);
#pragma unroll
        for (int z = 0; z < 8; ++z) {
            m = fmaxf(m, fabsf(x[z]));
            lds[i * D + d + z] = x[z];
        }
    }
    m = block_max(m, red);
    sc = fmaxf(vs0, m / 127.0f);
    y = 1.0f / sc;
    const float ratio = s0 && sc > vs0 ? vs0 / sc : 1.0f;
    // groups of 16 slots of one channel, from the first that holds a new token or,
    // where the scale grew, an old one
    const int g0 = ratio < 1.0f ? 0 : s0 / 16, g1 = (s1 + 15) / 16;
    for (int e = tid; e < (g1 - g0) * D; e += kThreads) {
        const int d = e % D, g = g0 + e / D;
        v4i* at = reinterpret_cast<v4i*>(vc + (int64_t)d * a.page + g * 16);
        v4i w{0, 0, 0, 0};
        if (g * 16 < s0 || g * 16 + 16 > s1) w = *at;
        float x[16];
#pragma unroll
        for (int z = 0; z < 16; ++z) {
            const int slot = g * 16 + z;
            x[z] = slot >= s0 && slot < s1 ? lds[(slot - s0) * D + d] : 0.0f;
        }
        uint32_t c[4];
        codes16(x, sc, y, c);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t was = (uint32_t)w[q], low = rescale4(was, ratio);
            uint32_t r = 0;
#pragma unroll
            for (int z = 0; z < 4; ++z) {
                const int slot = g * 16 + 4 * q + z;
                const uint32_t pick = slot < s0 ? low : slot < s1 ? c[q] : was;
                r |= pick & (255u << (8 * z));
            }
            w[q] = (int)r;
        }
        *at = w;
    }
    if (tid == 0) a.v_scale[ph] = sc;
}

// Workgroups [0, blocks): pages of one key head each; the rest rotate the queries,
// one thread per unit of `per` heads of a token.
template <int VEC>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(AppendArgs a, RopeArgs qa, int64_t blocks, int per) {
    extern __shared__ __attribute__((aligned(16))) float lds[];
    __shared__ float red[kThreads / kWave];
    if ((int64_t)blockIdx.x < blocks) {
        append_block<VEC>(a, blockIdx.x / a.heads, (int)(blockIdx.x % a.heads), lds, red);
        return;
    }
    const int units = qa.D / (2 * VEC), groups = (qa.H + per - 1) / per;
    const int64_t e = ((int64_t)blockIdx.x - blocks) * kThreads + threadIdx.x;
    const int u = (int)(e % units);
    const int64_t tg = e / units;
    const int g = (int)(tg % groups);
    if (tg / groups >= a.T) return;
    const int t = (int)(tg / groups);
    // the token's sequence: rows outside every sequence are left as they were
    const int b = find_seq(a.cu, a.B, a.T, t, 1, 1, 0);
    const Seq s = load_seq(a.cu, a.lens, b, a.T, a.max_pages * a.page);
    if (t < s.t0 || t >= s.t0 + s.n) return;
    const int h0 = g * per;
    rotate_unit<VEC>(qa, t, a.pos ? a.pos[t] : s.off + (t - s.t0), h0, min(per, qa.H - h0), u);
}

// ---- pages back as values ------------------------------------------------------------------------------------

// One workgroup: one listed page of one head, keys and values as [token][D] fp16.
__global__ __launch_bounds__(kThreads) void kv_read_kernel(const int8_t* __restrict__ k, const int8_t* __restrict__ v,
                                                           const float* __restrict__ k_scale,
                                                           const float* __restrict__ v_scale, int pages, int page,
                                                           int heads, int D, const int32_t* __restrict__ list,
                                                           uint16_t* __restrict__ Ko, uint16_t* __restrict__ Vo) {
    const int h = blockIdx.x % heads;
    const int64_t i = blockIdx.x / heads;
    const int pid = list[i];
    const bool there = (uint32_t)pid < (uint32_t)pages;
    const int64_t ph = there ? (int64_t)pid * heads + h : 0;
    const int8_t *kc = k + ph * page * D, *vc = v + ph * page * D;
    const float ks = k_scale[ph], vs = v_scale[ph];
    uint16_t *ko = Ko + (i * heads + h) * page * D, *vo = Vo + (i * heads + h) * page * D;
    for (int e = threadIdx.x; e < page * D / 8; e += kThreads) {
        const int tok = e / (D / 8), d = e % (D / 8) * 8;
        float x[8], y[8];
#pragma unroll
        for (int z = 0; z < 8; ++z) {
            x[z] = there ? (float)kc[e * 8 + z] * ks : 0.0f;
            y[z] = there ? (float)vc[(d + z) * page + tok] * vs : 0.0f;
        }
        store_run<8>(ko + e * 8, x);
        store_run<8>(vo + e * 8, y);
    }
}

// Heads of one token that a thread rotates: one while that leaves the card short of
// threads, so that a step's few tokens spread over it; eight past that, which share
// the angles.
int heads_per_thread(int64_t units) { return units > 256 * 1024 ? 8 : 1; }

int64_t rope_blocks(const RopeArgs& a, int vec, int per) {
    const int64_t threads = (int64_t)a.T * ((a.H + per - 1) / per) * (a.D / (2 * vec));
    return (threads + kThreads - 1) / kThreads;
}

}  // namespace

hipError_t launch_rope_frequencies(int rot, double base, int scaling, double factor, double original, double beta_fast,
                                   double beta_slow, double* freq, hipStream_t st) {
    hipLaunchKernelGGL(rope_frequencies_kernel, dim3((rot / 2 + kThreads - 1) / kThreads), dim3(kThreads), 0, st, rot,
                       base, scaling, factor, original, beta_fast, beta_slow, freq);
    return hipGetLastError();
}

hipError_t launch_rope(const uint16_t* X, int64_t x_token, int64_t x_head, const int32_t* pos, const double* freq, int T,
                       int H, int D, int rot, int layout, bool transpose, float amp, uint16_t* Y, int64_t y_token,
                       int64_t y_head, hipStream_t st) {
    const RopeArgs a{X, x_token, x_head, Y, y_token, y_head, freq, T, H, D, rot, layout, transpose, amp};
    if (rot % 16 == 0) {
        const int per = heads_per_thread((int64_t)T * H * (D / 16));
        hipLaunchKernelGGL(rope_kernel<8>, dim3((unsigned)rope_blocks(a, 8, per)), dim3(kThreads), 0, st, a, pos, per);
    } else {
        const int per = heads_per_thread((int64_t)T * H * (D / 2));
        hipLaunchKernelGGL(rope_kernel<1>, dim3((unsigned)rope_blocks(a, 1, per)), dim3(kThreads), 0, st, a, pos, per);
    }
    return hipGetLastError();
}

hipError_t launch_kv_append(int8_t* k, int8_t* v, float* k_scale, float* v_scale, int pages, int page, int heads, int D,
                            const uint16_t* K, int64_t k_token, int64_t k_head, const uint16_t* V, int64_t v_token,
                            int64_t v_head, const int32_t* cu, const int32_t* lens, const int32_t* table,
                            const int32_t* pos, int T, int B, int max_pages, const double* freq, int rot, int layout,
                            float amp, const uint16_t* Q, int64_t q_token, int64_t q_head, int Hq, uint16_t* Qr,
                            int64_t r_token, int64_t r_head, hipStream_t st) {
    const AppendArgs a{k, v, k_scale, v_scale, pages, page, heads, D, K, V, k_token, k_head, v_token, v_head,
                       cu, lens, table, pos, T, B, max_pages, freq, rot, layout, amp};
    const RopeArgs qa{Q, q_token, q_head, Qr, r_token, r_head, freq, T, Hq, D, rot, layout, false, amp};
    const int64_t blocks = touched_slots(T, B, page) * heads;
    const int bytes = page * D * (int)sizeof(float);
    static std::atomic<int> set8[kMaxDevices], set1[kMaxDevices];
    const bool wide = rot % 16 == 0;
    const hipError_t e = wide ? allow_dynamic_lds(reinterpret_cast<const void*>(&kv_append_kernel<8>), 128 << 10, set8)
                              : allow_dynamic_lds(reinterpret_cast<const void*>(&kv_append_kernel<1>), 128 << 10, set1);
    if (e != hipSuccess) return e;
    const int vec = wide ? 8 : 1;
    const int per = Q ? heads_per_thread((int64_t)T * Hq * (D / (2 * vec))) : 1;
    const int64_t grid = blocks + (Q ? rope_blocks(qa, vec, per) : 0);
    if (wide)
        hipLaunchKernelGGL(kv_append_kernel<8>, dim3((unsigned)grid), dim3(kThreads), bytes, st, a, qa, blocks, per);
    else
        hipLaunchKernelGGL(kv_append_kernel<1>, dim3((unsigned)grid), dim3(kThreads), bytes, st, a, qa, blocks, per);
    return hipGetLastError();
}

hipError_t launch_kv_read(const int8_t* k, const int8_t* v, const float* k_scale, const float* v_scale, int pages,
                          int page, int heads, int D, const int32_t* list, int n, uint16_t* Ko, uint16_t* Vo,
                          hipStream_t st) {
    hipLaunchKernelGGL(kv_read_kernel, dim3((unsigned)((int64_t)n * heads)), dim3(kThreads), 0, st, k, v, k_scale,
                       v_scale, pages, page, heads, D, list, Ko, Vo);
    return hipGetLastError();
}

}  // namespace sq
