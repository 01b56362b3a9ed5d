// Attention over the paged 8-bit cache for many rows of a key head: a workgroup turns
// a step's codes to halves once, in LDS, for all of its rows.
#include "attn_common.hpp"

namespace sq {
namespace {

typedef float f16v __attribute__((ext_vector_type(16)));

constexpr float kLargest = 11.0f, kMost = 15.0f;    // log2 of a row's largest weight: set to, and let grow to

// LDS of the tile kernel: two buffers of a step's keys [64][DP], two of its values
// [DP][64], as halves.  16-byte chunks of a row are swapped by the row so that 16
// lanes reading one chunk of 16 rows take 16 different bank groups.
template <int DP>
struct TileLds {
    static constexpr int kKeys = 64 * DP * 2;          // bytes of a buffer, of values too
    static __device__ __forceinline__ int key_at(int key, int chunk) {
        return key * (DP * 2) + ((chunk ^ (DP == 64 ? (key >> 1) & 7 : key & 15)) * 16);
    }
    static __device__ __forceinline__ int value_at(int d, int chunk) {
        return d * 128 + ((chunk ^ ((d >> 1) & 7)) * 16);
    }
};

// An offset whose uses are recomputed where they are: the other chunks of a row are an
// exclusive or away, which costs less than a register each.
__device__ __forceinline__ int here(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

__device__ __forceinline__ float lane_float(float x, int lane) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
}

template <int I>
struct Int {
    static constexpr int value = I;
};

// One workgroup of four waves has a tile of 128 rows, 32 a wave, whose queries stay in
// registers.  The matrix instruction is 32 x 32 x 16: an accumulator of S^T has keys
// 8 (i / 4) + 4 half + i % 4 of a tile of 32, and values are laid in LDS in that
// order.  While a step is multiplied the next one's codes become halves in the other
// buffer and those of the one after are requested: one barrier a step.
//
// WIDE: a page holds a step (64 or 128 tokens), so a step has one page and one pair of
// scales; otherwise each block of 16 keys has its own.
//
// Bound by the matrix cores and by what shares their waves' issue slots: 8 prompts of up
// to 2048 tokens (28 heads of 128 to 4) 400 to 430 us with the card's clock, 740 to 790
// TFLOP/s, against 1127 of a large library product.  In a series at 400 us the conversions
// of the codes cost 50, the loads 28, the exponentials 22 and the maximum 5 (copies that
// leave them out).  A tile's begin and end take as long as six of its steps: a sequence, its
// page, its codes, one after the other.  All 256 registers are in use: tiles of 128 channels
// keep 39 more in memory (56 for small pages), outside the loop over keys; those of 256 some
// 320, with about 30 loads a step in the loop, and are still ahead of tiles of 16 rows (206 us
// against 266 for 4 x 1024 tokens of 256 channels).
template <int DP, bool WIDE>
__global__ __launch_bounds__(256, DP <= 128 ? 2 : 1) void attn_tile_kernel(AttnArgs p) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    typedef TileLds<DP> L;
    constexpr int KS = DP / 16, DT = DP / 32, N = DP / 64;   // k steps, value tiles, 16-byte loads a thread of each
    constexpr int Z = WIDE ? 1 : 4;                          // scales a step
    constexpr int kAhead = 4;                                // operands read ahead
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int c = lane % 32, half = lane / 32;
    const int G = p.a.G, D = p.D, R = p.a.rows;
    const Group first = load_group(p, 0, lane);
    const Survey all = survey(p, first, lane);
    Share sh{};
    Tile tile{};
    const int worker = worker_of(p, all, 0, 1);
    if (!attn_always_direct(p.a) && blockIdx.x == 0 && threadIdx.x == 0) store_global(p.shared, (int)!all.direct);
    if (all.direct) {
        const int64_t tiles = gridDim.x / p.a.heads;
        const int64_t at = xcd_worker(blockIdx.x, gridDim.x);
        const int64_t item = attn_spread(at % tiles, tiles, attn_head_xcds(p.a.heads));
        if (at / tiles >= p.a.heads) return;
        const Listed l = find_listed(p, item, first, lane);
        const int64_t r64 = item - list_start(l.q.s.t0, l.b, G, R, 1);
        if (r64 < 0 || r64 >= l.q.tiles) return;
        const int r = l.q.slope < 0 ? (int)r64 : l.q.tiles - 1 - (int)r64;       // the longest first
        const AttnSteps steps = attn_steps(p.a, l.q.s, r);
        tile = {l.q.s, l.b, (int)(at / tiles), r,
                {0, steps.first, steps.first + steps.count, true, false, false}};
    } else {
        if ((int)blockIdx.x >= p.a.groups) return;
        if (tid == 0) store_global(p.lasts + worker, -1);
        sh = find_share(p, all.total, first, worker, lane);
    }
    for (;;) {
        if (!all.direct && !next_tile<false>(p, first, sh, worker, tile)) return;
        const Seq seq{__builtin_amdgcn_readfirstlane(tile.s.t0), __builtin_amdgcn_readfirstlane(tile.s.n),
                      __builtin_amdgcn_readfirstlane(tile.s.len), __builtin_amdgcn_readfirstlane(tile.s.off)};
        const AttnPart& part = tile.part;
        const int h = __builtin_amdgcn_readfirstlane(tile.h);
        const int rows = seq.n * G, row = tile.r * R + wave * 32 + c, at_row = min(row, rows - 1);
        const int pos = seq.off + at_row / G, qh = h * G + at_row % G, t = seq.t0 + at_row / G;
        const int lo = attn_lo(p.a, pos), hi = attn_hi(p.a, seq, pos);
        int lo_most = lo, hi_least = hi;               // of the wave's rows
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            lo_most = max(lo_most, __shfl_xor(lo_most, o, kWave));
            hi_least = min(hi_least, __shfl_xor(hi_least, o, kWave));
        }
        lo_most = __builtin_amdgcn_readfirstlane(lo_most);
        hi_least = __builtin_amdgcn_readfirstlane(hi_least);
        h8 Q[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int d = 16 * s + 8 * half;
            const uint16_t* q = p.Q + t * p.q_token + qh * p.q_head;
            Q[s] = d < D ? flip_query(load_query(q + d), p.flip) : h8{};
        }
        f16v O[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) O[d] = f16v{};
        float m = kUnseen, l = 0.0f;
        const int s0 = __builtin_amdgcn_readfirstlane(part.k0), s1 = __builtin_amdgcn_readfirstlane(part.k1);

        // 64 page table entries, one a lane, from entry `first_id` on, so that a step finds its
        // pages without a load of its own to wait for
        const int32_t* table = p.table + (int64_t)tile.b * p.max_pages;
        const int held = (seq.len + p.page - 1) >> p.shift;
        int ids = -1, first_id = -kWave;
        auto hold_pages = [&](int kt) {
            const int at = kt * kAttnStep >> p.shift;
            if (at + (WIDE ? 1 : kAttnStep >> p.shift) - first_id > kWave) {
                first_id = at;
                const int id = at + lane < held ? table[at + lane] : -1;
                ids = (uint32_t)id < (uint32_t)p.pages ? id : -1;
            }
        };
        auto head_of = [&](int pid) { return pid >= 0 ? (int64_t)pid * p.a.heads + h : (int64_t)h; };

        // this thread's part of a step, N pieces of 16 codes; past a head's channels it reads
        // others again, which meet zero queries or end in rows that are not stored; and the
        // scales of block lane % 4
        v4i kw[N], vw[N];
        float sk[2], sv[2];
        bool sin[2];
        auto fetch = [&](int kt, auto parity) {
            constexpr int A = decltype(parity)::value;
            hold_pages(kt);
            const int key0 = kt * kAttnStep, at = (key0 >> p.shift) - first_id;
            if constexpr (WIDE) {
                const int pid = __builtin_amdgcn_readlane(ids, at), slot = key0 & (p.page - 1);
                const int64_t ph = head_of(pid);
                const int8_t* kb = p.k + (ph * p.page + slot) * D;
                const int8_t* vb = p.v + ph * p.page * D + slot;
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    const int e = tid + 256 * n;
                    kw[n] = *reinterpret_cast<const v4i*>(
                        kb + (uint32_t)(e / (DP / 16) * D + min(e % (DP / 16) * 16, D - 16)));
                }
#pragma unroll
                for (int n = 0; n < N; ++n)
                    vw[n] = *reinterpret_cast<const v4i*>(
                        vb + (uint32_t)(min(tid / 4 + 64 * n, D - 1) * p.page + tid % 4 * 16));
                sin[A] = pid >= 0;
                sk[A] = p.k_scale[ph];
                sv[A] = p.v_scale[ph];
            } else {
                auto lane_page = [&](int key) { return __shfl(ids, at + (key >> p.shift), kWave); };
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    const int e = tid + 256 * n, key = e / (DP / 16), d = min(e % (DP / 16) * 16, D - 16);
                    kw[n] = *reinterpret_cast<const v4i*>(
                        p.k + (head_of(lane_page(key)) * p.page + (key & (p.page - 1))) * D + d);
                }
                const int u = tid % 4 * 16;
                const int8_t* vb = p.v + head_of(lane_page(u)) * D * p.page + (u & (p.page - 1));
#pragma unroll
                for (int n = 0; n < N; ++n)
                    vw[n] = *reinterpret_cast<const v4i*>(vb + (uint32_t)(min(tid / 4 + 64 * n, D - 1) * p.page));
                const int pid = lane_page(lane % 4 * 16);
                sin[A] = pid >= 0;
                sk[A] = p.k_scale[head_of(pid)];
                sv[A] = p.v_scale[head_of(pid)];
            }
        };
        // piece z / 2 of this thread's keys (z < 2 N) or values, its half z % 2, as halves into a buffer
        auto place = [&](uint8_t* keys, uint8_t* values, int k0, int v0, int z) {
            if (z < 2 * N) {
                // 256 pieces on: a multiple of 16 rows, which share their exchange of chunks
                const int n = z / 2, k = k0 + 256 * 16 / DP * n * (DP * 2);
                *reinterpret_cast<h8*>(keys + (k ^ (z % 2 * 16))) =
                    to_halves((uint32_t)kw[n][z % 2 * 2], (uint32_t)kw[n][z % 2 * 2 + 1]);
            } else {
                const int n = z / 2 - N, v = v0 + 64 * n * 128;      // 64 channels on
                *reinterpret_cast<h8*>(values + (v ^ (z % 2 * 16))) =
                    to_halves((uint32_t)vw[n][z % 2], (uint32_t)vw[n][z % 2 + 2]);
            }
        };
        auto step = [&](auto parity, auto last, int kt) {
            constexpr int A = decltype(parity)::value;
            constexpr bool kLast = decltype(last)::value;
            uint8_t *const keys = lds + A * L::kKeys, *const values = lds + (2 + A) * L::kKeys;
            BlockScale bs[Z];
            {
                const BlockScale k = block_scale(sin[A], sk[A], sv[A], p.scale);
#pragma unroll
                for (int z = 0; z < Z; ++z) bs[z] = {lane_float(k.ks, z), lane_float(k.lv, z), lane_float(k.iv, z)};
            }
            // First product, two tiles of 32 keys.  Operands are read kAhead instructions ahead;
            // the second tile's run beside the next step's codes becoming halves.  Barriers to
            // the scheduler hold this order: left to itself it reads an operand, waits and multiplies.
            f16v S[2];
            h8 K[kAhead];
            const int k0 = here(L::key_at(c, half));
            auto key_operand = [&](int i) {
                return *reinterpret_cast<const h8*>(keys + i / KS * 32 * (DP * 2) + (k0 ^ (32 * (i % KS))));
            };
#pragma unroll
            for (int i = 0; i < kAhead; ++i) K[i] = key_operand(i);
            __builtin_amdgcn_sched_barrier(0);
            const int kp = here(L::key_at(tid / (DP / 16), tid % (DP / 16) * 2));
            const int vp = here(L::value_at(tid / 4, tid % 4 * 2));
#pragma unroll
            for (int i = 0; i < 2 * KS; ++i) {
                S[i / KS] = __builtin_amdgcn_mfma_f32_32x32x16_f16(K[i % kAhead], Q[i % KS],
                                                                  i % KS ? S[i / KS] : f16v{}, 0, 0, 0);
                if (i + kAhead < 2 * KS) K[i % kAhead] = key_operand(i + kAhead);
                if (!kLast && i >= KS) place(lds + (A ^ 1) * L::kKeys, lds + (2 + (A ^ 1)) * L::kKeys, kp, vp, i - KS);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (!kLast) fetch(min(kt + 2, s1 - 1), parity);
            h8 V[2][DT];
            const int v0 = here(L::value_at(c, half));
#pragma unroll
            for (int d = 0; d < DT; ++d) V[0][d] = *reinterpret_cast<const h8*>(values + 32 * d * 128 + v0);
            __builtin_amdgcn_sched_barrier(0);

            const int key0 = kt * kAttnStep;
            if (key0 < lo_most || key0 + kAttnStep > hi_least) {
                int key = key0 + 4 * half;
                asm volatile("" : "+v"(key));          // keeps these comparisons out of the steps without an edge
                const uint32_t from = lo - key, span = hi > lo ? hi - lo : 0;
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if ((uint32_t)(32 * y + 8 * (e / 4) + e % 4) - from >= span) S[y][e] = kHidden;
            }
            float mx = kNone;
#pragma unroll
            for (int z = 0; z < 4; z += 4 / Z) {
                float bm = S[z / 2][8 * (z % 2)];
#pragma unroll
                for (int e = 1; e < 32 / Z; ++e) bm = fmaxf(bm, S[z / 2 + e / 16][(8 * (z % 2) + e) % 16]);
                const BlockScale& k = bs[z * Z / 4];
                mx = fmaxf(mx, __builtin_fmaf(bm, k.ks, k.lv));
            }
            mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
            if (__any(fabsf(mx) > kFine)) {
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    const BlockScale& k = bs[e / 8 * Z / 4];
                    S[e / 16][e % 16] = __builtin_fmaf(S[e / 16][e % 16], k.ks, k.lv);
                }
#pragma unroll
                for (int z = 0; z < Z; ++z) bs[z].ks = 1.0f, bs[z].lv = 0.0f;
            }
            // the reference follows once the largest weight would pass 2^15, so that the
            // accumulators are rescaled a few times a row
            if (__any(mx - m > kMost)) {
                const float mn = fmaxf(m, fabsf(mx) > kFine ? mx : mx - kLargest);
                const float fade = __builtin_amdgcn_exp2f(m - mn);
                m = mn;
                l *= fade;
#pragma unroll
                for (int d = 0; d < DT; ++d) O[d] *= fade;
            }
            // Second product, 16 keys at a time: the next 16 weights and operands beside the
            // instructions of these
            float sum = 0.0f;
            h8 W[2];
            auto weights = [&](int u, int e) {         // two of them
                const BlockScale& k = bs[u * Z / 4];
                const float off = k.lv - m;
                const int i = 8 * u + e;
                const f2 w = {__builtin_amdgcn_exp2f(__builtin_fmaf(S[i / 16][i % 16], k.ks, off)),
                              __builtin_amdgcn_exp2f(__builtin_fmaf(S[i / 16][i % 16 + 1], k.ks, off))};
                sum += w[0];
                sum += w[1];
                const h2 x = __builtin_convertvector(w, h2);
                W[u % 2][e] = x[0];
                W[u % 2][e + 1] = x[1];
                if (e == 6 && (Z > 1 || u == 3)) {
                    l = __builtin_fmaf(sum, k.iv, l);
                    sum = 0.0f;
                }
            };
#pragma unroll
            for (int e = 0; e < 8; e += 2) weights(0, e);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    if (u < 3)
                        V[(u + 1) % 2][d] =
                            *reinterpret_cast<const h8*>(values + 32 * d * 128 + (v0 ^ (32 * (u + 1))));
                    O[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(V[u % 2][d], W[u % 2], O[d], 0, 0, 0);
                    if (u < 3) {
#pragma unroll
                        for (int e = 0; e < 8; e += 2)
                            if (e * DT / 8 == d) weights(u + 1, e);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            if (!kLast) __syncthreads();
        };
        if (s0 < s1) {
            __syncthreads();                           // the tile before is done with the buffers
            fetch(s0, Int<0>());
#pragma unroll
            for (int z = 0; z < 4 * N; ++z)
                place(lds, lds + 2 * L::kKeys, L::key_at(tid / (DP / 16), tid % (DP / 16) * 2),
                      L::value_at(tid / 4, tid % 4 * 2), z);
            fetch(min(s0 + 1, s1 - 1), Int<1>());
            __syncthreads();
            int kt = s0;
            for (; kt + 2 < s1; kt += 2) {
                step(Int<0>(), Int<0>(), kt);
                step(Int<1>(), Int<0>(), kt + 1);
            }
            if (kt + 1 < s1) {
                step(Int<0>(), Int<0>(), kt);
                step(Int<1>(), Int<1>(), kt + 1);
            } else {
                step(Int<0>(), Int<1>(), kt);
            }
        }
        l += __shfl_xor(l, 32, kWave);
        const bool none = s0 < s1 && l == 0.0f && lo < hi;
        if (__any(none)) {                             // products of -inf, where a query is infinite
            h8 q[KS];
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int d = 16 * s + 8 * half;
                q[s] = d < D ? load_query(p.Q + t * p.q_token + qh * p.q_head + d) : h8{};
            }
            float fault = query_fault(q);
            fault += __shfl_xor(fault, 32, kWave);
            if (none) l = fault;
        }
        if (row < rows) {
            const int64_t o = (int64_t)t * p.a.heads * G + qh;
            const int lr = wave * 32 + c;
            const float inv = inverse(m, l);
            const bool split = part.begins_inside || part.ends_inside, any = s0 < s1 && !part.whole;
            float* ws = p.places + attn_place(worker, part.begins_inside) * attn_place_floats(R, D);
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int ch = 32 * d + 8 * e + 4 * half;
                    const f4 x{O[d][4 * e], O[d][4 * e + 1], O[d][4 * e + 2], O[d][4 * e + 3]};
                    if (ch < D) {
                        if (part.whole) store_result(p.O + o * D + ch, x, inv);
                        else if (any) store_global(ws + lr * D + ch, x);
                    }
                }
            if (half == 0) {
                if (split) {
                    store_global(ws + R * D + lr, any ? m : kNone);
                    store_global(ws + R * D + R + lr, l);
                }
                if (part.whole && p.lse) store_global(p.lse + o, result_lse(m, l));
            }
        }
        if (all.direct) return;
    }
}

template <int DP>
hipError_t launch(const AttnArgs& p, hipStream_t st) {
    constexpr int bytes = 4 * TileLds<DP>::kKeys;
    static std::atomic<int> wide_set[kMaxDevices], set[kMaxDevices];
    const bool wide = p.page >= kAttnStep;
    const hipError_t e =
        wide ? allow_dynamic_lds(reinterpret_cast<const void*>(&attn_tile_kernel<DP, true>), bytes, wide_set)
             : allow_dynamic_lds(reinterpret_cast<const void*>(&attn_tile_kernel<DP, false>), bytes, set);
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)attn_grid(p.a));
    if (wide)
        hipLaunchKernelGGL((attn_tile_kernel<DP, true>), grid, dim3(256), bytes, st, p);
    else
        hipLaunchKernelGGL((attn_tile_kernel<DP, false>), grid, dim3(256), bytes, st, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_tile(const AttnArgs& p, hipStream_t st) {
    return p.D <= 64 ? launch<64>(p, st) : p.D <= 128 ? launch<128>(p, st) : launch<256>(p, st);
}

}  // namespace sq
