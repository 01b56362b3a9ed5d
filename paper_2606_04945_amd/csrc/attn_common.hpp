// Attention over the paged 8-bit cache: what its kernels share.
//
// out = sum_j w_j v_j with w = softmax(scale q . k_j) over the visible keys, one
// pass over the keys in steps of 64.  Codes go to the fp16 matrix cores as they
// are, every int8 being an fp16; a page's key scale multiplies its logits in fp32.
// Its value scale s goes into the weight: with x the logit times log2 e,
//   w = 2^(x + log2 s - m),  O = sum w code,  l = sum w / s,  out = O / l,
// and m a running reference below the largest x + log2 s, so that a weight is rounded
// to fp16 relative to the row's largest contribution however the scales differ, and
// the rounding of log2 s cancels between O and l.  Where the reference rises to m', O
// and l are multiplied by 2^(m - m').  How far below: fp16 holds weights from 2^-14 on
// with 11 bits, smaller ones with half a step of 2^-25, and a row whose largest weight
// meets small values consists of its small weights.  So the largest is near the upper
// end, at 2^14 in tiles of 16 and 32 rows, between 2^11 and 2^15 in those of 128, whose
// reference may lag: half a step is 2^-39 and 2^-36 of it.
//
// Both products are formed transposed, S^T = K Q^T and O^T = V^T P^T: a lane then
// has one query's logits, which are where the second product wants that query's
// weights, if the keys of a step are dealt to matrix rows so that both agree.
// Softmax weights never leave their lane, and keys ([token][D]) and values
// ([D][token]) are row operands as they are stored.
#pragma once
#include "attn_plan.hpp"
#include "tile_common.hpp"

namespace sq {

struct AttnArgs {
    AttnShape a;
    const uint16_t* Q;
    int64_t q_token, q_head;
    const int8_t *k, *v;
    const float *k_scale, *v_scale;
    int pages, page, shift, D;      // page = 1 << shift
    const int32_t *cu, *lens, *table;
    int max_pages;
    float scale;                    // its magnitude, times log2 e
    uint32_t flip;                  // sign bits of a pair of halves where the scale is negative
    uint16_t* O;
    float* lse;
    int *shared, *lasts;            // of the workspace: whether tiles are shared; a worker's last worker,
    AttnRecord* records;            // its record, its places
    float* places;
};

hipError_t launch_attn_wave(const AttnArgs& p, hipStream_t st);
hipError_t launch_attn_tile(const AttnArgs& p, hipStream_t st);

namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNone = -__builtin_inff();

// Stores through pointers that are known to be global.  From a pointer of no known
// space the compiler makes a flat store, and while one may be pending every wait for a
// load is a wait for all loads: the loops over keys would have none in flight.
template <class T>
__device__ __forceinline__ void store_global(void* p, const T& x) {
    *(__attribute__((address_space(1))) T*)p = x;
}

// Sum over the lanes up to this one: shifts within rows of 16 lanes, then the rows'
// last lanes spread to the rows after them.
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t add_shifted(int64_t v) {
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, true);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)((uint64_t)v >> 32), CTRL, ROWS, 0xf, true);
    return v + (int64_t)(((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ int64_t wave_scan(int64_t v) {
    v = add_shifted<0x111, 0xf>(v);      // row_shr 1, 2, 4, 8
    v = add_shifted<0x112, 0xf>(v);
    v = add_shifted<0x114, 0xf>(v);
    v = add_shifted<0x118, 0xf>(v);
    v = add_shifted<0x142, 0xa>(v);      // lane 15 of a row to the next row, into rows 1 and 3
    return add_shifted<0x143, 0xc>(v);   // lane 31 into rows 2 and 3
}
__device__ __forceinline__ int64_t lane_value(int64_t v, int lane) {
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)v, lane);
    const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)v >> 32), lane);
    return (int64_t)(((uint64_t)hi << 32) | lo);
}

// 64 sequences of the batch, one a lane (none past the last: no rows).
struct Group {
    int c0, c1, len;
};
__device__ __forceinline__ Group load_group(const AttnArgs& p, int b0, int lane) {
    const int b = b0 + lane, at = min(b, p.a.B - 1);
    const Group g{p.cu[at], p.cu[at + 1], p.lens[at]};
    return b < p.a.B ? g : Group{p.a.T, p.a.T, 0};
}
__device__ __forceinline__ AttnSeq group_seq(const AttnArgs& p, const Group& g) {
    return attn_seq(p.a, g.c0, g.c1, g.len);
}
__device__ __forceinline__ AttnSeq lane_seq(const AttnArgs& p, const Group& g, int lane) {
    return attn_seq(p.a, __builtin_amdgcn_readlane(g.c0, lane), __builtin_amdgcn_readlane(g.c1, lane),
                    __builtin_amdgcn_readlane(g.len, lane));
}

// sequence b, the same for all lanes
__device__ __forceinline__ AttnSeq scalar_seq(const AttnArgs& p, int b) {
    return attn_seq(p.a, p.cu[b], p.cu[b + 1], p.lens[b]);
}

// What every workgroup works out first: the weight of all tiles, and whether the
// batch is read tile by tile.
struct Survey {
    int64_t total;
    bool direct;
};
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t max_shifted(int64_t v) {
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, true);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)((uint64_t)v >> 32), CTRL, ROWS, 0xf, true);
    return max(v, (int64_t)(((uint64_t)hi << 32) | lo));
}
__device__ __forceinline__ int64_t wave_max64(int64_t v) {   // of values >= 0
    v = max_shifted<0x111, 0xf>(v);
    v = max_shifted<0x112, 0xf>(v);
    v = max_shifted<0x114, 0xf>(v);
    v = max_shifted<0x118, 0xf>(v);
    v = max_shifted<0x142, 0xa>(v);
    return lane_value(max_shifted<0x143, 0xc>(v), kWave - 1);
}
__device__ __forceinline__ Survey survey(const AttnArgs& p, const Group& first, int lane) {
    if (attn_always_direct(p.a)) return {0, true};
    int64_t total = 0, most = 0;
    Group g = first;
    for (int b0 = 0;;) {
        const AttnSeq q = group_seq(p, g);
        total += lane_value(wave_scan(q.weight), kWave - 1);
        most = max(most, wave_max64(attn_most(q)));
        b0 += kWave;
        if (b0 >= p.a.B) break;
        g = load_group(p, b0, lane);
    }
    total *= p.a.heads;
    return {total, attn_direct(p.a, total, most)};
}

// A worker's part of the weight, [at, end), the sequence it begins in and the
// weight before that sequence.
struct Share {
    int64_t at, end, before;
    int b;
    AttnCut cut;
};
__device__ __forceinline__ Share find_share(const AttnArgs& p, int64_t total, const Group& first, int worker,
                                            int lane) {
    const int workers = attn_workers(p.a, total);
    const AttnCut cut = attn_cut_work(total, workers);
    if (worker >= workers) return {0, 0, 0, p.a.B, cut};
    Share s{attn_start(cut, worker), attn_start(cut, worker + 1), 0, p.a.B, cut};
    for (int b0 = 0; b0 < p.a.B; b0 += kWave) {
        const int64_t w = group_seq(p, b0 ? load_group(p, b0, lane) : first).weight, upto = wave_scan(w);
        const uint64_t past = __ballot(s.before + upto * p.a.heads > s.at);
        if (past) {
            const int i = __builtin_ctzll(past);
            s.b = b0 + i;
            s.before += lane_value(upto - w, i) * p.a.heads;
            break;
        }
        s.before += lane_value(upto, kWave - 1) * p.a.heads;
    }
    return s;
}

// The sequence whose list of tiles holds place `item`: the last whose list starts
// at or before it (list starts do not decrease).
struct Listed {
    int b;
    AttnSeq q;
};
__device__ __forceinline__ Listed find_listed(const AttnArgs& p, int64_t item, const Group& first, int lane) {
    Listed r{};
    Group g = first;
    for (int b0 = 0;;) {
        const int64_t start = list_start(min(max(g.c0, 0), p.a.T), b0 + lane, p.a.G, p.a.rows, 1);
        const bool at = b0 + lane < p.a.B && start <= item;
        const int n = __popcll(__ballot(at));
        if (n > 0) {
            r.b = b0 + n - 1;
            r.q = lane_seq(p, g, n - 1);
        }
        b0 += kWave;
        if (n < kWave || b0 >= p.a.B) return r;
        g = load_group(p, b0, lane);
    }
}

// Worker of a workgroup: dispatch goes round the XCDs, and neighbouring workers read
// the same keys, so each XCD gets a run of them.
__device__ __forceinline__ int xcd_worker(int L, int W) {
    const int x = L % kXcds, base = W / kXcds, rem = W % kXcds;
    return x * base + (x < rem ? x : rem) + L / kXcds;
}

// A wave's or a workgroup's worker: runs of them as above, or, where some have no part,
// the ones that do spread over the workgroups.
__device__ __forceinline__ int worker_of(const AttnArgs& p, const Survey& all, int wave, int waves) {
    if (attn_workers(p.a, all.total) < p.a.workers) return wave * p.a.groups + blockIdx.x;
    return xcd_worker(blockIdx.x, p.a.groups) * waves + wave;
}

// The tile at a worker's position and what it does of it; moves the position on, and
// leaves the record of a tile that goes on in a later worker's part.  False at the end.
struct Tile {
    Seq s;
    int b, h, r;
    AttnPart part;
};
template <bool LANES>      // sequences from the lanes that hold them, no load, for three registers
__device__ __forceinline__ bool next_tile(const AttnArgs& p, const Group& first, Share& sh, int worker, Tile& t) {
    while (sh.at < sh.end && sh.b < p.a.B) {
        const AttnSeq q = LANES && sh.b < kWave ? lane_seq(p, first, sh.b) : scalar_seq(p, sh.b);
        const int64_t weight = q.weight * p.a.heads;
        if (sh.at - sh.before >= weight) {             // also a sequence without rows
            sh.before += weight;
            ++sh.b;
            continue;
        }
        const int h = (int)divide(sh.at - sh.before, q.weight);
        const int r = attn_find_tile(q, sh.at - sh.before - h * q.weight);
        t = {q.s, sh.b, h, r, attn_part(p.a, q, sh.before, h, r, sh.at, sh.end)};
        sh.at = t.part.next;
        if (t.part.ends_inside && !t.part.begins_inside) {
            const int64_t past = sh.before + h * q.weight + attn_before(q, r) + q.base + q.slope * r;
            if (threadIdx.x % kWave == 0) {
                store_global(p.lasts + worker, attn_worker(sh.cut, past - 1));
                store_global(p.records + worker, v4i{q.s.t0, q.s.n * p.a.G, r * p.a.rows, h});
            }
        }
        return true;
    }
    return false;
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

// A hidden key's product, and the reference of a row that has seen no key: low, and
// finite, so that a hidden key's weight is 0 without a test.  A page whose scales are not
// finite numbers >= 0 has the logit kBad, which no others come near: a row that sees a key
// of it ends with that reference, and is NaN.
constexpr float kHidden = -__builtin_inff(), kUnseen = -0x1p126f, kBad = 0x1p120f;

// Logits of larger magnitude are rounded before the reference is subtracted from them, which
// takes an instruction more for each: the usual form subtracts it from the product itself,
// and where fp32 rounds logits by more than a bit or two the largest, which the reference was
// taken from, may be that much above it.  A reference there is the largest itself.
constexpr float kFine = 0x1p18f;

// What a block of 16 keys (one page) multiplies: logits by ks, and w by 2^lv with
// 1 / s = iv.  Keys of no page, or past the length, take no part: lv = -inf.  A value
// scale below 2^-60, 0 included, counts as that: its contribution to an fp16 result
// is 0 either way, and 2^28 weights of 2^15 times 2^60 have a sum in fp32.  The limits
// of the key scale keep its products finite, and above 0, so that a hidden key's stay -inf.
struct BlockScale {
    float ks, lv, iv;
};
__device__ __forceinline__ BlockScale block_scale(bool in, float ks, float vs, float scale) {
    constexpr int kNot = 0x001 | 0x002 | 0x004 | 0x008 | 0x010 | 0x200;     // classes: NaN, -inf, negative, inf
    const bool bad = __builtin_amdgcn_classf(ks, kNot) | __builtin_amdgcn_classf(vs, kNot);
    const float s = fminf(fmaxf(vs, 0x1p-60f), 0x1p100f), lv = bad ? kBad : __builtin_amdgcn_logf(s);
    return {in & !bad ? fminf(fmaxf(ks * scale, 1e-25f), 3e38f) : 1.0f, in ? lv : kNone, __builtin_amdgcn_rcpf(s)};
}

__device__ __forceinline__ h8 load_query(const uint16_t* q) {
    return __builtin_bit_cast(h8, *reinterpret_cast<const v4i*>(q));
}
// a negative scale's sign goes into the queries, so that larger products are larger logits
__device__ __forceinline__ h8 flip_query(h8 q, uint32_t flip) {
    return __builtin_bit_cast(h8, __builtin_bit_cast(v4i, q) ^ (int)flip);
}

// NaN if a query is not finite, else 0
template <int N>
__device__ __forceinline__ float query_fault(const h8 (&q)[N]) {
    h8 z{};
#pragma unroll
    for (int i = 0; i < N; ++i) z += q[i] * (_Float16)0.0f;
    return (float)(((z[0] + z[1]) + (z[2] + z[3])) + ((z[4] + z[5]) + (z[6] + z[7])));
}

// what a row's sums are multiplied by at the end: 0 of a row that has seen no key
__device__ __forceinline__ float inverse(float m, float l) {
    return l == 0.0f ? 0.0f : m < kBad / 2 ? 1.0f / l : __builtin_nanf("");
}

// four results of a row as fp16
__device__ __forceinline__ void store_result(uint16_t* o, f4 x, float inv) {
    const u32x2 w = {(uint32_t)f2h(x[0] * inv) | ((uint32_t)f2h(x[1] * inv) << 16),
                     (uint32_t)f2h(x[2] * inv) | ((uint32_t)f2h(x[3] * inv) << 16)};
    store_global(o, w);
}

__device__ __forceinline__ float result_lse(float m, float l) {
    return l == 0.0f ? kNone : m < kBad / 2 ? (m + __builtin_amdgcn_logf(l)) * kLn2 : __builtin_nanf("");
}

}  // namespace
}  // namespace sq
