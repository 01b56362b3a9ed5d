// Work division of the attention over the paged cache: index arithmetic shared by
// the kernels, the host and code without a GPU compiler.
//
// A sequence's query tokens, each with the G query heads of a key head, make rows
// (row = token G + head); BM rows of one key head are a tile, and a tile's visible
// keys are read KT at a time, a step.  Lengths live on the device, so the grid is a
// fixed number of workers, and each finds its share there: tiles are laid end to
// end in the order (sequence, key head, row tile), each with a weight close to its
// number of visible keys, and worker w takes the w-th equal part of the sum.  A
// part that ends inside a tile takes that fraction of its steps.  A tile whose
// steps all fall to one worker is written by it; of the others every worker leaves
// a partial result, and a second kernel joins them.
//
// Weights only balance the load: tile r of a sequence weighs base + slope r, a
// closed form that needs no loop over tiles.
#pragma once
#include "kv_plan.hpp"

namespace sq {

constexpr int kAttnStep = 64;     // keys per step

struct AttnShape {
    int T, B, heads, G;           // query rows, sequences, key heads, query heads per key head
    int max_len;                  // positions a page table row holds
    int causal, window;
    int rows;                     // rows per tile
    int workers;
};

struct AttnSeq {
    Seq s;
    int tiles;                    // row tiles per key head
    int64_t base, slope, weight;  // of tile r: base + slope r; of one key head: the sum
};

SQ_HD AttnSeq attn_seq(const AttnShape& a, int c0, int c1, int len) {
    AttnSeq q;
    q.s = make_seq(c0, c1, len, a.T, a.max_len);
    q.tiles = (int)(((int64_t)q.s.n * a.G + a.rows - 1) / a.rows);
    if (a.causal && !a.window) {
        q.slope = a.rows;
        q.base = (int64_t)a.G * ((q.s.off > 0 ? q.s.off : 0) + kAttnStep) + a.rows;
    } else {
        const int64_t reach = (int64_t)a.window + a.rows / a.G + 1;
        const int64_t span = a.window && reach < q.s.len ? reach : q.s.len;
        q.slope = 0;
        q.base = a.G * (span + kAttnStep);
    }
    q.weight = q.tiles * q.base + q.slope * ((int64_t)q.tiles * (q.tiles - 1) / 2);
    return q;
}

// Weight of the tiles before tile r of one key head.
SQ_HD int64_t attn_before(const AttnSeq& q, int r) { return r * q.base + q.slope * ((int64_t)r * (r - 1) / 2); }

// The tile of one key head that weight position x (0 <= x < q.weight) falls in.
SQ_HD int attn_find_tile(const AttnSeq& q, int64_t x) {
    int lo = 0, hi = q.tiles - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (attn_before(q, mid) <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// Keys that a query at position p sees: [lo, hi), empty where hi <= lo.
SQ_HD int attn_lo(const AttnShape& a, int p) {
    const int64_t lo = (int64_t)p - a.window + 1;
    return a.window && lo > 0 ? (int)(lo < 0x7fffffff ? lo : 0x7fffffff) : 0;
}
SQ_HD int attn_hi(const AttnShape& a, const Seq& s, int p) {
    return !a.causal || p + 1 > s.len ? s.len : p + 1 > 0 ? p + 1 : 0;
}

// Steps that the rows of tile r read: [first, first + count).
struct AttnSteps {
    int first, count;
};
SQ_HD AttnSteps attn_steps(const AttnShape& a, const Seq& s, int r) {
    const int64_t row0 = (int64_t)r * a.rows, end = (int64_t)s.n * a.G;
    const int64_t last = row0 + a.rows < end ? row0 + a.rows - 1 : end - 1;
    const int lo = attn_lo(a, s.off + (int)(row0 / a.G)), hi = attn_hi(a, s, s.off + (int)(last / a.G));
    if (hi <= lo) return {0, 0};
    return {lo / kAttnStep, (hi + kAttnStep - 1) / kAttnStep - lo / kAttnStep};
}

// Weight positions of worker w: [attn_start(w), attn_start(w + 1)).
SQ_HD int64_t attn_start(int64_t total, int workers, int w) {
    const int64_t q = total / workers, rem = total % workers;
    return w * q + (w < rem ? w : rem);
}
// The worker whose part holds position x.
SQ_HD int attn_worker(int64_t total, int workers, int64_t x) {
    const int64_t q = total / workers, rem = total % workers;
    return (int)(x < rem * (q + 1) ? x / (q + 1) : rem + (x - rem * (q + 1)) / q);
}

// Of `count` steps of a tile of weight `weight`, those before fraction x / weight.
// 0 at 0 and count at weight, so the parts of a tile cover its steps once.
SQ_HD int attn_cut(int64_t x, int64_t weight, int count) {
    return x <= 0 ? 0 : x >= weight ? count : (int)((x * count + weight - 1) / weight);
}

// Partial results: two places for each worker, the tile its part begins inside of
// and the tile it ends inside of.  A place holds, per row, D sums in fp32, the
// maximum and the sum of the row's softmax.
SQ_HD int attn_place(int w, bool begins_inside) { return 2 * w + (begins_inside ? 0 : 1); }
SQ_HD int64_t attn_place_floats(int rows, int D) { return (int64_t)rows * (D + 2); }

// Tiles of all sequences and key heads, at most: what the joining kernel's grid covers.
inline int64_t attn_tile_slots(const AttnShape& a) { return ((int64_t)a.T * a.G / a.rows + a.B) * a.heads; }

// Workers that a call starts: as many as run at once, fewer where the steps cannot
// be that many.
inline int attn_workers(const AttnShape& a, int at_once) {
    const int64_t steps = ((int64_t)a.max_len + kAttnStep - 1) / kAttnStep;
    const int64_t tiles = attn_tile_slots(a);
    const int64_t most = tiles > at_once ? at_once : tiles * (steps > 0 ? steps : 1);
    return (int)(most < 1 ? 1 : most < at_once ? most : at_once);
}

constexpr int kAttnWaves = 256 * 8;      // one-wave workers: two for each SIMD of 256 CUs

}  // namespace sq
