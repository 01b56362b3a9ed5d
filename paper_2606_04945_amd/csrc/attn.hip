// Attention over the paged 8-bit cache: which kernel a call takes, and the kernel that
// joins partial results.
#include "attn_common.hpp"
#include "serve.hpp"

namespace sq {
namespace {

// Joins the partial results of the tiles that workers share:
//   out = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i.
// Every workgroup finds the shared tiles in the workers' entries; tiles times parts of
// their rows go round the workgroups, as many parts as make that one each, so that a few
// tiles of many results and many of few both spread over the card.  A group of D / 4
// threads has a row, four channels a thread; where a workgroup has more groups than rows,
// several share a row's results and meet in LDS in order.  Which worker ended first
// changes nothing.  Bound by three round trips to memory that other XCDs wrote and, for
// tiles of 128 rows, by the partial results' bytes (32 next tokens of 28 heads
// 6.5 us, 2 x 512 tokens 15 us, 4 where nothing is shared).  Twice the workgroups: no change.
constexpr int kJoinThreads = 256, kJoinGroups = 64;    // at most: heads of 16
constexpr int kJoinBlocks = 512, kJoinMasks = kAttnCus * 8 / kWave;
__global__ __launch_bounds__(kJoinThreads) void attn_join_kernel(AttnArgs p) {
    __shared__ uint64_t masks[kJoinMasks];
    __shared__ float ml[2 * kJoinGroups];
    __shared__ f4 part[kJoinThreads];
    const int tid = threadIdx.x, R = p.a.rows, D = p.D, G = p.a.G;
    const int vecs = D / 4, groups = kJoinThreads / vecs, gi = tid / vecs, v = tid % vecs;
    const int lane = tid % kWave, wave = tid / kWave;
    const int64_t size = attn_place_floats(R, D);
    // 64 workers a mask, a bit each: a tile that others end
    int last[kJoinMasks / 4];
#pragma unroll
    for (int i = 0; i < kJoinMasks / 4; ++i) last[i] = p.lasts[min(i * kJoinThreads + tid, p.a.workers - 1)];
    if (!*p.shared) return;
#pragma unroll
    for (int i = 0; i < kJoinMasks / 4; ++i) {
        const uint64_t found = __ballot(i * kJoinThreads + tid < p.a.workers && last[i] >= 0);
        if (lane == 0) masks[i * 4 + wave] = found;
    }
    __syncthreads();
    const uint64_t mask = lane < kJoinMasks ? masks[lane] : 0;
    const int upto = (int)wave_scan(__popcll(mask)), tiles = __builtin_amdgcn_readlane(upto, kWave - 1);
    if (tiles == 0) return;
    const int parts = min(R, max(1, kJoinBlocks / tiles));
    for (int item = blockIdx.x; item < tiles * parts; item += kJoinBlocks) {
        const int k = item / parts, first = item % parts;      // rows first, first + parts, ...
        const int at_mask = __builtin_ctzll(__ballot(upto > k));
        uint64_t bits = (uint64_t)lane_value((int64_t)mask, at_mask);
        for (int z = k - (__builtin_amdgcn_readlane(upto, at_mask) - __popcll(bits)); z > 0; --z) bits &= bits - 1;
        const int w0 = at_mask * kWave + __builtin_ctzll(bits), n = p.lasts[w0] - w0 + 1;
        const AttnRecord t = p.records[w0];
        const int rows = (min(R, t.rows - t.row0) - first + parts - 1) / parts;
        if (rows <= 0) continue;
        const int per = min(n, max(1, groups / rows));         // groups of threads to a row
        for (int r0 = 0; r0 < rows; r0 += groups / per) {
            const int row = first + (r0 + gi / per) * parts;
            const bool in = gi < groups / per * per && r0 + gi / per < rows;
            float m = kNone, l = 0.0f;
            f4 O{0, 0, 0, 0};
            if (in) {
                constexpr int U = 4;                   // results requested together
                for (int j0 = gi % per; j0 < n; j0 += U * per) {
                    float mj[U], lj[U];
                    f4 Oj[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int j = j0 + u * per, w = w0 + min(j, n - 1);
                        const float* ws = p.places + attn_place(w, w > w0) * size;
                        mj[u] = j < n ? ws[R * D + row] : kNone;
                        lj[u] = ws[R * D + R + row];
                        Oj[u] = *reinterpret_cast<const f4*>(ws + row * D + 4 * v);
                    }
                    float mn = m;
#pragma unroll
                    for (int u = 0; u < U; ++u) mn = fmaxf(mn, mj[u]);
                    const float ms = fmaxf(mn, kUnseen);                 // -inf: nothing yet
                    const float f = __builtin_amdgcn_exp2f(m - ms);
                    O *= f;
                    l *= f;
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        // a place without a maximum holds no sums either
                        const bool some = mj[u] != kNone;
                        const float fu = __builtin_amdgcn_exp2f(mj[u] - ms);
#pragma unroll
                        for (int i = 0; i < 4; ++i) O[i] = some ? __builtin_fmaf(Oj[u][i], fu, O[i]) : O[i];
                        l = some ? __builtin_fmaf(lj[u], fu, l) : l;
                    }
                    m = mn;
                }
            }
            if (per > 1) {
                __syncthreads();
                part[tid] = O;
                if (v == 0 && gi < groups) ml[gi] = m, ml[kJoinGroups + gi] = l;
                __syncthreads();
                if (in && gi % per == 0)
                    for (int z = 1; z < per; ++z) {
                        const float mz = ml[gi + z], mn = fmaxf(m, mz), ms = fmaxf(mn, kUnseen);
                        const float f = __builtin_amdgcn_exp2f(m - ms), fz = __builtin_amdgcn_exp2f(mz - ms);
                        O = O * f + part[tid + z * vecs] * fz;
                        l = l * f + ml[kJoinGroups + gi + z] * fz;
                        m = mn;
                    }
            }
            if (!in || gi % per || m == kNone) continue;      // no maximum: one worker wrote the row
            const int at = t.row0 + row;
            const int64_t o = (int64_t)(t.t0 + at / G) * p.a.heads * G + t.h * G + at % G;
            store_result(p.O + o * D + 4 * v, O, inverse(m, l));
            if (p.lse && v == 0) store_global(p.lse + o, result_lse(m, l));
        }
    }
}

}  // namespace

size_t attn_workspace_bytes(int T, int B, int Hq, int heads, int D, int max_len) {
    return (size_t)attn_workspace_most(T, B, Hq, heads, D, max_len);
}

hipError_t launch_attn(const uint16_t* Q, int64_t q_token, int64_t q_head, const int8_t* k, const int8_t* v,
                       const float* k_scale, const float* v_scale, int pages, int page, int heads, int D,
                       const int32_t* cu, const int32_t* lens, const int32_t* table, int T, int B, int max_pages, int Hq,
                       bool causal, int window, float scale, uint16_t* O, float* lse, void* ws, hipStream_t st) {
    const AttnShape a = attn_shape(T, B, Hq, heads, D, max_pages * page, causal, window);
    int *shared = static_cast<int*>(ws), *lasts = shared + 4;
    AttnRecord* records = reinterpret_cast<AttnRecord*>(lasts + a.workers);
    const AttnArgs p{a, Q, q_token, q_head, k, v, k_scale, v_scale, pages, page, __builtin_ctz((unsigned)page), D,
                     cu, lens, table, max_pages, fabsf(scale) * kLog2e, scale < 0.0f ? 0x80008000u : 0u, O, lse,
                     shared, lasts, records, reinterpret_cast<float*>(records + a.workers)};
    const hipError_t e = a.rows > 32 ? launch_attn_tile(p, st) : launch_attn_wave(p, st);
    if (e != hipSuccess || attn_always_direct(a)) return e;
    hipLaunchKernelGGL(attn_join_kernel, dim3(kJoinBlocks), dim3(kJoinThreads), 0, st, p);
    return hipGetLastError();
}

}  // namespace sq
