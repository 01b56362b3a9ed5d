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

// One thread: one unit of `per` heads of one token.  Bound by its bytes where there are
// many (16384 tokens of 28 heads of 128: 44 us, 5.4 TB/s, as fast as a copy) and by a
// launch and two round trips where there are few (16 tokens of 32 heads: 3.4 us).
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

// The batch's first 64 sequences, one a lane of the wave.
struct Lanes {
    int c0, c1, len;
};
__device__ __forceinline__ Lanes load_lanes(const AppendArgs& a, int b0, int lane) {
    const int b = b0 + lane, at = min(b, a.B - 1);
    const Lanes l{a.cu[at], a.cu[at + 1], a.lens[at]};
    return b < a.B ? l : Lanes{a.T, a.T, 0};
}
__device__ __forceinline__ Seq lane_seq(const AppendArgs& a, const Lanes& l, int lane) {
    return make_seq(__builtin_amdgcn_readlane(l.c0, lane), __builtin_amdgcn_readlane(l.c1, lane),
                    __builtin_amdgcn_readlane(l.len, lane), a.T, a.max_pages * a.page);
}

// The sequence whose list of touched pages holds place `item`, by one wave: the last
// whose list starts at or before it.
__device__ __forceinline__ int find_page(const AppendArgs& a, int64_t item, int lane, Seq& s) {
    int b = 0;
    for (int b0 = 0; b0 < a.B; b0 += kWave) {
        const Lanes l = load_lanes(a, b0, lane);
        const bool at = b0 + lane < a.B && list_start(min(max(l.c0, 0), a.T), b0 + lane, 1, a.page, 2) <= item;
        const int n = __popcll(__ballot(at));
        if (n > 0) {
            b = b0 + n - 1;
            s = lane_seq(a, l, n - 1);
        }
        if (n < kWave) break;
    }
    return b;
}

// The sequence of row t, another one for each lane: the last that starts at or before
// it.  Up to 64 sequences are compared from the lanes' own, more by halving.
__device__ __forceinline__ Seq find_row(const AppendArgs& a, int t, int lane) {
    if (a.B <= kWave) {
        const Lanes l = load_lanes(a, 0, lane);
        int n = 0;
        for (int b = 0; b < a.B; ++b) n += min(max(__builtin_amdgcn_readlane(l.c0, b), 0), a.T) <= t;
        const int at = max(n - 1, 0);
        return make_seq(__shfl(l.c0, at, kWave), __shfl(l.c1, at, kWave), __shfl(l.len, at, kWave), a.T,
                        a.max_pages * a.page);
    }
    int lo = 0, hi = a.B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (min(max(a.cu[mid], 0), a.T) <= t) lo = mid; else hi = mid - 1;
    }
    return make_seq(a.cu[lo], a.cu[lo + 1], a.lens[lo], a.T, a.max_pages * a.page);
}

// The new tokens of one page: slots [s0, s1), whose first is row `row` at position `pos`.
struct Span {
    int s0, s1, row, pos, pid;
    int64_t ph;
};

// The larger of two values, NaN if one is: a page must not lose what went wrong upstream.
__device__ __forceinline__ float largest(float x, float y) { return __builtin_elementwise_maximum(x, y); }

// largest over the workgroup of two values at once
__device__ __forceinline__ void block_max(float& x, float& y, float* red) {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) {
        x = largest(x, __shfl_xor(x, o, kWave));
        y = largest(y, __shfl_xor(y, o, kWave));
    }
    if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = x, red[kThreads / kWave + threadIdx.x / kWave] = y;
    __syncthreads();
    x = red[0], y = red[kThreads / kWave];
#pragma unroll
    for (int w = 1; w < kThreads / kWave; ++w) {
        x = largest(x, red[w]);
        y = largest(y, red[kThreads / kWave + w]);
    }
}

// A page's scale from its old one and the new magnitudes' largest: NaN if not finite.
__device__ __forceinline__ float page_scale(float old, float most) {
    const float s = largest(old, most / 127.0f);
    return s < __builtin_inff() ? s : __builtin_nanf("");
}

// codes of 8 values against scale s, y = 1 / s, a byte each; zero codes for s = 0 or NaN
__device__ __forceinline__ void codes8(const float* x, float s, float y, uint32_t& lo, uint32_t& hi) {
    int c[8];
    quant_codes8<127>(x, s, y, c);
    auto word = [&](int q) {
        return (uint32_t)(c[q] & 255) | ((uint32_t)(c[q + 1] & 255) << 8) | ((uint32_t)(c[q + 2] & 255) << 16) |
               ((uint32_t)c[q + 3] << 24);
    };
    lo = word(0), hi = word(4);
    if (!(s > 0.0f)) lo = hi = 0;
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

// Older codes of the page under a larger scale: code' = rint(code s / s').
__device__ __forceinline__ void rescale_keys(int8_t* kc, int count, float ratio) {
    for (int e = threadIdx.x; e < count / 4; e += kThreads) {
        uint32_t* w = reinterpret_cast<uint32_t*>(kc) + e;
        *w = rescale4(*w, ratio);
    }
}

// The values' codes, [D][page / 4 + 1] words of four slots in LDS, into the page: 16
// slots of a channel at a time, from the first group that holds a new token or, where the
// scale grew, an old one.  Bytes of other slots come from memory.
__device__ __forceinline__ void store_values(int8_t* vc, const uint32_t* words, const Span& p, int page, int D,
                                             float ratio) {
    const int g0 = ratio < 1.0f ? 0 : p.s0 / 16, groups = (p.s1 + 15) / 16 - g0;
    for (int e = threadIdx.x; e < groups * D; e += kThreads) {
        const int g = g0 + e % groups, d = e / groups;
        v4i* at = reinterpret_cast<v4i*>(vc + d * page + g * 16);
        const bool mixed = g * 16 < p.s0 || g * 16 + 16 > p.s1;
        v4i w{0, 0, 0, 0};
        if (mixed) w = *at;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t fresh = words[d * (page / 4 + 1) + g * 4 + q];
            if (!mixed) {
                w[q] = (int)fresh;
                continue;
            }
            const uint32_t was = (uint32_t)w[q], low = ratio < 1.0f ? rescale4(was, ratio) : was;
            uint32_t r = 0;
#pragma unroll
            for (int z = 0; z < 4; ++z) {
                const int slot = g * 16 + 4 * q + z;
                r |= (slot < p.s0 ? low : slot < p.s1 ? fresh : was) & (255u << (8 * z));
            }
            w[q] = (int)r;
        }
        *at = w;
    }
}

// Rotated keys and the values of a page in registers: KU units of 2 x 8 key entries and
// VI blocks of 4 slots x 8 value channels a thread.  Everything the page's tokens bring
// is requested before the page's old scales are waited for, the largest magnitudes of
// both are found together, and the codes go out as they are formed, the values' through
// LDS, where they change from tokens to channels.  Prompts are bound by their bytes (11300
// tokens of 28 + 4 + 4 heads of 128, the queries among them: 39 us, 5.0 TB/s), a step's
// few tokens by four round trips in a row: batch, page table, scales, older codes (9 us).
template <int KU, int VI>
__device__ void append_registers(const AppendArgs& a, const Span& p, int h, uint32_t* words, float* red) {
    const int D = a.D, tid = threadIdx.x, n = p.s1 - p.s0, units = D / 16, channels = D / 8;
    v4i ka[KU], kb[KU], vv[VI][4];
#pragma unroll
    for (int u = 0; u < KU; ++u) {
        const int e = tid + kThreads * u, i = e / units;
        const RopeUnit r = rope_unit<8>(e % units, a.rot, a.layout);
        const uint16_t* x = a.K + (p.row + i) * a.k_token + h * a.k_head;
        ka[u] = i < n ? *reinterpret_cast<const v4i*>(x + r.a) : v4i{0, 0, 0, 0};
        kb[u] = i < n ? *reinterpret_cast<const v4i*>(x + r.b) : v4i{0, 0, 0, 0};
    }
#pragma unroll
    for (int u = 0; u < VI; ++u) {
        const int e = tid + kThreads * u, slot = (p.s0 / 4 + e / channels) * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = slot + j - p.s0;
            const uint16_t* x = a.V + (p.row + i) * a.v_token + h * a.v_head + e % channels * 8;
            vv[u][j] = i >= 0 && i < n ? *reinterpret_cast<const v4i*>(x) : v4i{0, 0, 0, 0};
        }
    }
    const float ks0 = p.s0 ? a.k_scale[p.ph] : 0.0f, vs0 = p.s0 ? a.v_scale[p.ph] : 0.0f;
    float x[KU][16], km = 0.0f, vm = 0.0f;
#pragma unroll
    for (int u = 0; u < KU; ++u) {
        const int e = tid + kThreads * u, i = e / units;
        const RopeUnit r = rope_unit<8>(e % units, a.rot, a.layout);
        float xa[8], xb[8];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            xa[2 * q] = h2f((uint16_t)(uint32_t)ka[u][q]), xa[2 * q + 1] = h2f((uint16_t)((uint32_t)ka[u][q] >> 16));
            xb[2 * q] = h2f((uint16_t)(uint32_t)kb[u][q]), xb[2 * q + 1] = h2f((uint16_t)((uint32_t)kb[u][q] >> 16));
        }
        if (r.pair >= 0 && i < n) {
            const int pos = a.pos ? a.pos[p.row + i] : p.pos + i;
            float c[8], s[8];
#pragma unroll
            for (int z = 0; z < 8; ++z) rope_angle(pos, a.freq[r.pair + z], a.amp, false, c[z], s[z]);
            rope_turn<8>(xa, xb, c, s, a.layout);
        }
#pragma unroll
        for (int z = 0; z < 8; ++z) {
            x[u][z] = xa[z], x[u][8 + z] = xb[z];
            km = largest(km, largest(fabsf(xa[z]), fabsf(xb[z])));
        }
    }
#pragma unroll
    for (int u = 0; u < VI; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                vm = largest(vm, largest(fabsf(h2f((uint16_t)(uint32_t)vv[u][j][q])),
                                         fabsf(h2f((uint16_t)((uint32_t)vv[u][j][q] >> 16)))));
    block_max(km, vm, red);
    const float ks = page_scale(ks0, km), ky = 1.0f / ks, vs = page_scale(vs0, vm), vy = 1.0f / vs;
    if (tid == 0) a.k_scale[p.ph] = ks, a.v_scale[p.ph] = vs;
    int8_t *kc = a.k + p.ph * a.page * D, *vc = a.v + p.ph * a.page * D;
    if (p.s0 && ks > ks0) rescale_keys(kc, p.s0 * D, ks0 / ks);
#pragma unroll
    for (int u = 0; u < KU; ++u) {
        const int e = tid + kThreads * u, i = e / units;
        if (i >= n) continue;
        const RopeUnit r = rope_unit<8>(e % units, a.rot, a.layout);
        uint2 w;
        codes8(x[u], ks, ky, w.x, w.y);
        *reinterpret_cast<uint2*>(kc + (p.s0 + i) * D + r.a) = w;
        codes8(x[u] + 8, ks, ky, w.x, w.y);
        *reinterpret_cast<uint2*>(kc + (p.s0 + i) * D + r.b) = w;
    }
#pragma unroll
    for (int u = 0; u < VI; ++u) {
        const int e = tid + kThreads * u, slot = (p.s0 / 4 + e / channels) * 4;
        if (slot >= p.s1) continue;
        uint32_t lo[4], hi[4];                         // of the four slots: channels 0 .. 3, 4 .. 7
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float y[8];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                y[2 * q] = h2f((uint16_t)(uint32_t)vv[u][j][q]);
                y[2 * q + 1] = h2f((uint16_t)((uint32_t)vv[u][j][q] >> 16));
            }
            codes8(y, vs, vy, lo[j], hi[j]);
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            uint32_t w = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) w |= ((q < 4 ? lo[j] : hi[j]) >> (8 * (q % 4)) & 255u) << (8 * j);
            words[(e % channels * 8 + q) * (a.page / 4 + 1) + slot / 4] = w;
        }
    }
    __syncthreads();
    store_values(vc, words, p, a.page, D, p.s0 && vs > vs0 ? vs0 / vs : 1.0f);
}

// The same for a rotated part that does not divide into units of 2 x 8: the rotated keys
// wait in LDS, [token][D] fp32, a pair at a time.
__device__ void append_pairs(const AppendArgs& a, const Span& p, int h, float* lds, float* red) {
    const int D = a.D, tid = threadIdx.x, n = p.s1 - p.s0, units = D / 2;
    const float ks0 = p.s0 ? a.k_scale[p.ph] : 0.0f, vs0 = p.s0 ? a.v_scale[p.ph] : 0.0f;
    float km = 0.0f, vm = 0.0f;
    for (int e = tid; e < n * units; e += kThreads) {
        const int i = e / units;
        const uint16_t* x = a.K + (p.row + i) * a.k_token + h * a.k_head;
        const RopeUnit r = rope_unit<1>(e % units, a.rot, a.layout);
        float u[1] = {h2f(x[r.a])}, v[1] = {h2f(x[r.b])};
        if (r.pair >= 0) {
            float c[1], s[1];
            rope_angle(a.pos ? a.pos[p.row + i] : p.pos + i, a.freq[r.pair], a.amp, false, c[0], s[0]);
            rope_turn<1>(u, v, c, s, a.layout);
        }
        km = largest(km, largest(fabsf(u[0]), fabsf(v[0])));
        lds[i * D + r.a] = u[0];
        lds[i * D + r.b] = v[0];
    }
    for (int e = tid; e < n * D; e += kThreads)
        vm = largest(vm, fabsf(h2f(a.V[(p.row + e / D) * a.v_token + h * a.v_head + e % D])));
    block_max(km, vm, red);
    const float ks = page_scale(ks0, km), ky = 1.0f / ks, vs = page_scale(vs0, vm), vy = 1.0f / vs;
    if (tid == 0) a.k_scale[p.ph] = ks, a.v_scale[p.ph] = vs;
    int8_t *kc = a.k + p.ph * a.page * D, *vc = a.v + p.ph * a.page * D;
    if (p.s0 && ks > ks0) rescale_keys(kc, p.s0 * D, ks0 / ks);
    for (int e = tid; e < n * D / 8; e += kThreads) {
        float x[8];
#pragma unroll
        for (int z = 0; z < 8; ++z) x[z] = lds[e * 8 + z];
        uint2 w;
        codes8(x, ks, ky, w.x, w.y);
        *reinterpret_cast<uint2*>(kc + p.s0 * D + e * 8) = w;
    }
    __syncthreads();                                   // the keys are out of LDS
    uint32_t* words = reinterpret_cast<uint32_t*>(lds);
    for (int e = tid; e < (p.s1 / 4 - p.s0 / 4 + 1) * D; e += kThreads) {
        const int d = e % D, slot = (p.s0 / 4 + e / D) * 4;
        if (slot >= p.s1) continue;
        float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = slot + j - p.s0;
            if (i >= 0 && i < n) x[j] = h2f(a.V[(p.row + i) * a.v_token + h * a.v_head + d]);
        }
        uint32_t lo, hi;
        codes8(x, vs, vy, lo, hi);
        words[d * (a.page / 4 + 1) + slot / 4] = lo;
    }
    __syncthreads();
    store_values(vc, words, p, a.page, D, p.s0 && vs > vs0 ? vs0 / vs : 1.0f);
}

// Workgroups [0, blocks): a page of one key head each, whose codes of that head they
// own; the rest rotate the queries, a thread one unit of `per` heads of a token.
// KU 0: the rotated part does not divide into units of 2 x 8 entries.
template <int KU>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(AppendArgs a, RopeArgs qa, int64_t blocks, int per) {
    extern __shared__ __attribute__((aligned(16))) float lds[];
    __shared__ float red[2 * kThreads / kWave];
    const int lane = threadIdx.x % kWave;
    if ((int64_t)blockIdx.x < blocks) {
        const int64_t item = blockIdx.x / a.heads;
        const int h = blockIdx.x % a.heads;
        Seq s{0, 0, 0, 0};
        const int b = find_page(a, item, lane, s);
        const int64_t j = item - list_start(s.t0, b, 1, a.page, 2);
        if (j < 0 || j >= touched_count(s, a.page)) return;
        const int blk = touched_first(s, a.page) + (int)j;
        const int pid = a.table[(int64_t)b * a.max_pages + blk];
        if ((uint32_t)pid >= (uint32_t)a.pages) return;
        const int p0 = max(s.off, blk * a.page), p1 = min(s.len, (blk + 1) * a.page);   // positions written
        const Span p{p0 - blk * a.page, p1 - blk * a.page, s.t0 + p0 - s.off, p0, pid, (int64_t)pid * a.heads + h};
        if constexpr (KU > 0)
            append_registers<KU, (KU + 1) / 2>(a, p, h, reinterpret_cast<uint32_t*>(lds), red);
        else
            append_pairs(a, p, h, lds, red);
        return;
    }
    constexpr int VEC = KU > 0 ? 8 : 1;
    const int units = qa.D / (2 * VEC), groups = (qa.H + per - 1) / per;
    const int64_t e = ((int64_t)blockIdx.x - blocks) * kThreads + threadIdx.x;
    const int u = (int)(e % units);
    const int64_t tg = e / units;
    const int g = (int)(tg % groups);
    const int t = (int)min(tg / groups, (int64_t)a.T);
    // the token's sequence: rows outside every sequence are left as they were
    const Seq s = find_row(a, t, lane);
    if (t >= a.T || t < s.t0 || t >= s.t0 + s.n) return;
    const int h0 = g * per;
    rotate_unit<VEC>(qa, t, a.pos ? a.pos[t] : s.off + (t - s.t0), h0, min(per, qa.H - h0), u);
}

// ---- pages back as values ------------------------------------------------------------------------------------

// One workgroup: one listed page of one head, keys and values as [token][D] fp16.  The
// values' codes pass through LDS, where 4 x 4 blocks of bytes change their order; a
// padded row keeps the reads of consecutive channels off each other's banks.  Bound by
// its stores: 732 pages and heads of 64 x 128 in 8.2 us, 4.4 TB/s.
__global__ __launch_bounds__(kThreads) void kv_read_kernel(const int8_t* __restrict__ k, const int8_t* __restrict__ v,
                                                           const float* __restrict__ k_scale,
                                                           const float* __restrict__ v_scale, int pages, int page,
                                                           int heads, int D, const int32_t* __restrict__ list,
                                                           uint16_t* __restrict__ Ko, uint16_t* __restrict__ Vo) {
    extern __shared__ __attribute__((aligned(16))) uint32_t codes[];    // [D][page / 4 + 1]
    const int h = blockIdx.x % heads, tid = threadIdx.x;
    const int64_t i = blockIdx.x / heads;
    const int pid = list[i];
    const bool there = (uint32_t)pid < (uint32_t)pages;
    const int64_t ph = there ? (int64_t)pid * heads + h : 0;
    const int size = page * D, words = page / 4, row = words + 1;
    const v4i *kc = reinterpret_cast<const v4i*>(k + ph * size), *vc = reinterpret_cast<const v4i*>(v + ph * size);
    const float ks = there ? k_scale[ph] : 0.0f, vs = there ? v_scale[ph] : 0.0f;
    uint16_t *ko = Ko + (i * heads + h) * size, *vo = Vo + (i * heads + h) * size;
    for (int e = tid; e < size / 16; e += kThreads) {
        const v4i w = vc[e];
        const int at = e / (words / 4) * row + e % (words / 4) * 4;
#pragma unroll
        for (int q = 0; q < 4; ++q) codes[at + q] = (uint32_t)w[q];
    }
    for (int e = tid; e < size / 16; e += kThreads) {
        const v4i w = kc[e];
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            float x[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) x[q] = there ? (float)(int8_t)(w[2 * z + q / 4] >> (8 * (q % 4))) * ks : 0.0f;
            store_run<8>(ko + e * 16 + 8 * z, x);
        }
    }
    __syncthreads();
    for (int e = tid; e < words * (D / 4); e += kThreads) {      // four tokens of four channels
        const int d = e % (D / 4) * 4, t = e / (D / 4);
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = codes[(d + q) * row + t];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            float x[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) x[q] = there ? (float)(int8_t)(w[q] >> (8 * s)) * vs : 0.0f;
            uint2 y;
            y.x = (uint32_t)f2h(x[0]) | ((uint32_t)f2h(x[1]) << 16);
            y.y = (uint32_t)f2h(x[2]) | ((uint32_t)f2h(x[3]) << 16);
            *reinterpret_cast<uint2*>(vo + (4 * t + s) * D + d) = y;
        }
    }
}

// Heads of one token that a thread rotates: one while that leaves the card short of
// threads, so that a step's few tokens spread over it; eight past that, which share
// the angles.  32 heads of 128, one / eight (us): 512 tokens 4.5 / 6.4, 1024 tokens
// 6.5 / 8.1, 2048 tokens 10.5 / 9.5; appending 8 x 512 tokens 32.2 / 24.5.
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
    const bool wide = rot % 16 == 0;
    const int vec = wide ? 8 : 1;
    const int per = Q ? heads_per_thread((int64_t)T * Hq * (D / (2 * vec))) : 1;
    const dim3 grid((unsigned)(blocks + (Q ? rope_blocks(qa, vec, per) : 0)));
    if (!wide) {
        static std::atomic<int> set[kMaxDevices];
        const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(&kv_append_kernel<0>), 128 << 10, set);
        if (e != hipSuccess) return e;
        const int keys = page * D * (int)sizeof(float), values = D * (page + 4);
        hipLaunchKernelGGL(kv_append_kernel<0>, grid, dim3(kThreads), keys > values ? keys : values, st, a, qa, blocks,
                           per);
        return hipGetLastError();
    }
    const int bytes = D * (page + 4), units = (page * (D / 16) + kThreads - 1) / kThreads;   // units a thread
    if (units <= 1)
        hipLaunchKernelGGL(kv_append_kernel<1>, grid, dim3(kThreads), bytes, st, a, qa, blocks, per);
    else if (units <= 2)
        hipLaunchKernelGGL(kv_append_kernel<2>, grid, dim3(kThreads), bytes, st, a, qa, blocks, per);
    else if (units <= 4)
        hipLaunchKernelGGL(kv_append_kernel<4>, grid, dim3(kThreads), bytes, st, a, qa, blocks, per);
    else
        hipLaunchKernelGGL(kv_append_kernel<8>, grid, dim3(kThreads), bytes, st, a, qa, blocks, per);
    return hipGetLastError();
}

hipError_t launch_kv_read(const int8_t* k, const int8_t* v, const float* k_scale, const float* v_scale, int pages,
                          int page, int heads, int D, const int32_t* list, int n, uint16_t* Ko, uint16_t* Vo,
                          hipStream_t st) {
    hipLaunchKernelGGL(kv_read_kernel, dim3((unsigned)((int64_t)n * heads)), dim3(kThreads), D * (page + 4), st, k, v,
                       k_scale, v_scale, pages, page, heads, D, list, Ko, Vo);
    return hipGetLastError();
}

}  // namespace sq
