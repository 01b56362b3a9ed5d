// Attention over the paged 8-bit cache: which kernel a call takes, and the kernel that
// joins partial results.
#include "attn_common.hpp"

namespace sq {
namespace {

// Joins the partial results of a tile: out = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i.
// A workgroup has `share` rows of one tile.  A group of `vecs` threads has a row,
// four channels a thread; where the results are many, several groups share a row's,
// and meet in LDS in order.  Which worker ended first changes nothing.
constexpr int kJoinThreads = 256, kJoinPlaces = 2048, kJoinAtOnce = 256 * 8;
__global__ __launch_bounds__(kJoinThreads) void attn_join_kernel(AttnArgs p, int share) {
    __shared__ int places[kJoinPlaces];
    __shared__ int counts[kJoinThreads / kWave];
    __shared__ float ml[2 * kJoinThreads];
    __shared__ f4 part[kJoinThreads];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int R = p.a.rows, D = p.D, G = p.a.G;
    const int64_t item = blockIdx.x / p.a.heads;
    const int h = blockIdx.x % p.a.heads;
    const Group first = load_group(p, 0, lane);
    const Survey all = survey(p, first, lane);
    if (all.direct) return;
    const Listed at_item = find_listed<true>(p, item, first, lane);
    const AttnSeq q = at_item.q;
    const int64_t r64 = item - list_start(q.s.t0, at_item.b, G, R, 1);
    if (r64 < 0 || r64 >= q.tiles) return;
    const int r = (int)r64, row0 = blockIdx.y * share;
    const int rows = min(min(R, row0 + share), q.s.n * G - r * R);
    if (row0 >= rows) return;
    const AttnSteps steps = attn_steps(p.a, q.s, r);
    if (steps.count <= 1) return;                 // never split
    const int64_t before = at_item.before;
    const AttnCut cut = attn_cut_work(all.total, p.a.workers);
    const int64_t from = before + h * q.weight + attn_before(q, r), weight = q.base + q.slope * r;
    const int w0 = attn_worker(cut, from), w1 = attn_worker(cut, from + weight - 1);
    if (w0 == w1) return;
    int n = 0;                                    // results, in the workers' order
    for (int wb = w0; wb <= w1; wb += kJoinThreads) {
        const int w = wb + tid;
        int place = -1;
        bool alone = false;
        if (w <= w1) {
            const int64_t x0 = attn_start(cut, w) - from, x1 = min(attn_start(cut, w + 1) - from, weight);
            const int k0 = attn_cut(x0, weight, steps.count), k1 = attn_cut(x1, weight, steps.count);
            alone = k1 - k0 == steps.count;
            if (k1 > k0) place = attn_place(w, x0 > 0);
        }
        if (__syncthreads_or(alone)) return;      // one worker had every step and wrote the rows
        const uint64_t some = __ballot(place >= 0);
        if (lane == 0) counts[wave] = __popcll(some);
        __syncthreads();
        int base = n;
#pragma unroll
        for (int v = 0; v < kJoinThreads / kWave; ++v) {
            if (v < wave) base += counts[v];
            n += counts[v];
        }
        if (place >= 0) places[base + __popcll(some & ((1ull << lane) - 1))] = place;
    }
    __syncthreads();
    const int vecs = D / 4, groups = kJoinThreads / vecs;
    const int each = min(n, max(1, groups / (rows - row0)));      // groups of threads to a row
    const int64_t size = attn_place_floats(R, D);
    const int gi = tid / vecs, v = tid % vecs;
    for (int first = row0; first < rows; first += groups / each) {
        const int row = first + gi / each;
        const bool mine = gi < groups && row < rows;
        float m = kUnseen, l = 0.0f;
        f4 O{0, 0, 0, 0};
        if (mine) {
            constexpr int U = 8;                  // results requested together
            for (int j0 = gi % each; j0 < n; j0 += U * each) {
                float mj[U], lj[U];
                f4 Oj[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int j = j0 + u * each;
                    const float* ws = p.ws + places[min(j, n - 1)] * size;
                    mj[u] = j < n ? ws[R * D + row] : kNone;
                    lj[u] = ws[R * D + R + row];
                    Oj[u] = *reinterpret_cast<const f4*>(ws + row * D + 4 * v);
                }
                float mn = m;
#pragma unroll
                for (int u = 0; u < U; ++u) mn = fmaxf(mn, mj[u]);
                const float f = __builtin_amdgcn_exp2f(m - mn);
                O *= f;
                l *= f;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const float fu = __builtin_amdgcn_exp2f(mj[u] - mn);
                    O += Oj[u] * fu;
                    l = __builtin_fmaf(lj[u], fu, l);
                }
                m = mn;
            }
        }
        if (each > 1) {
            __syncthreads();
            part[tid] = O;
            ml[tid] = m, ml[kJoinThreads + tid] = l;
            __syncthreads();
            if (!mine || gi % each) continue;
            for (int z = 1; z < each; ++z) {
                const int o = tid + z * vecs;
                const float mn = fmaxf(m, ml[o]);
                const float f = __builtin_amdgcn_exp2f(m - mn), fz = __builtin_amdgcn_exp2f(ml[o] - mn);
                O = O * f + part[o] * fz;
                l = l * f + ml[kJoinThreads + o] * fz;
                m = mn;
            }
        }
        if (!mine) continue;
        const int at = r * R + row;
        const int64_t o = (int64_t)(q.s.t0 + at / G) * p.a.heads * G + h * G + at % G;
        store_result(p.O + o * D + 4 * v, O, l > 0.0f ? 1.0f / l : 0.0f);
        if (p.lse && v == 0) p.lse[o] = result_lse(m, l);
    }
}

}  // namespace

size_t attn_workspace_bytes(int T, int B, int Hq, int heads, int D, int max_len) {
    const AttnShape a = attn_shape(T, B, Hq, heads, D, max_len, true, 0);
    return attn_always_direct(a) ? 0 : (size_t)a.workers * 2 * attn_place_floats(a.rows, D) * sizeof(float);
}

hipError_t launch_attn(const uint16_t* Q, int64_t q_token, int64_t q_head, const int8_t* k, const int8_t* v,
                       const float* k_scale, const float* v_scale, int pages, int page, int heads, int D,
                       const int32_t* cu, const int32_t* lens, const int32_t* table, int T, int B, int max_pages, int Hq,
                       bool causal, int window, float scale, uint16_t* O, float* lse, void* ws, hipStream_t st) {
    const AttnShape a = attn_shape(T, B, Hq, heads, D, max_pages * page, causal, window);
    const AttnArgs p{a, Q, q_token, q_head, k, v, k_scale, v_scale, pages, page, __builtin_ctz((unsigned)page), D,
                     cu, lens, table, max_pages, fabsf(scale) * kLog2e, scale < 0.0f ? 0x80008000u : 0u, O, lse,
                     static_cast<float*>(ws)};
    const hipError_t e = a.rows > 32 ? launch_attn_tile(p, st) : launch_attn_wave(p, st);
    if (e != hipSuccess || attn_always_direct(a)) return e;
    // rows a joining workgroup has: fewer while the workgroups still run all at once
    const int64_t tiles = attn_tile_slots(a);
    int share = a.rows;
    while (share > 1 && tiles * (a.rows / share) < kJoinAtOnce) share /= 2;
    hipLaunchKernelGGL(attn_join_kernel, dim3((unsigned)tiles, (unsigned)(a.rows / share)), dim3(kJoinThreads), 0,
                       st, p, share);
    return hipGetLastError();
}

}  // namespace sq
