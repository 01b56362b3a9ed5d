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
// closed form that needs no loop over tiles: its keys and a step's, within a factor of
// two of them with a window.
#pragma once
#include "kv_plan.hpp"

namespace sq {

constexpr int kAttnStep = 64;     // keys per step

// a / b for 0 <= a, 0 < b.  Weights of a usual batch fit 32 bits, where a division
// is several times as fast.
SQ_HD int64_t divide(int64_t a, int64_t b) {
    return ((uint64_t)a | (uint64_t)b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

struct AttnShape {
    int T, B, heads, G;           // query rows, sequences, key heads, query heads per key head
    int max_len;                  // positions a page table row holds
    int causal, window;
    int rows;                     // rows per tile
    int groups;                   // workgroups that run at once
    int workers;                  // workers that share the work where tiles are split
    int join;                     // keys whose reading takes as long as the joining kernel
};

struct AttnSeq {
    Seq s;
    int tiles;                    // row tiles per key head
    int64_t base, slope, weight;  // of tile r: base + slope r; of one key head: the sum
};

SQ_HD AttnSeq attn_seq(const AttnShape& a, int c0, int c1, int len) {
    AttnSeq q;
    q.s = make_seq(c0, c1, len, a.T, a.max_len);
    q.tiles = (q.s.n * a.G + a.rows - 1) / a.rows;      // T G is below 2^27
    if (a.causal && !a.window) {
        q.slope = a.rows;
        q.base = (int64_t)a.G * ((q.s.off > 0 ? q.s.off : 0) + kAttnStep) + a.rows;
    } else if (a.window && !a.causal) {
        // a query sees all later keys: the window's length and the tokens from its own on, but no
        // more than there are, which a line leaves out
        q.slope = -a.rows;
        q.base = a.G * ((int64_t)q.s.n + (a.window < q.s.len ? a.window : q.s.len) + kAttnStep);
    } else {
        const int64_t reach = (int64_t)a.window + a.rows / a.G + 1;
        const int64_t span = a.window && reach < q.s.len ? reach : q.s.len;
        q.slope = 0;
        q.base = a.G * (span + kAttnStep);
    }
    q.weight = q.tiles * q.base + q.slope * ((int64_t)q.tiles * (q.tiles - 1) / 2);
    return q;
}
// Weight of the largest tile.
SQ_HD int64_t attn_most(const AttnSeq& q) {
    return q.tiles > 0 ? q.base + (q.slope > 0 ? q.slope * (q.tiles - 1) : 0) : 0;
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
    const int row0 = r * a.rows, end = s.n * a.G;
    const int last = row0 + a.rows < end ? row0 + a.rows - 1 : end - 1;
    const int lo = attn_lo(a, s.off + row0 / a.G), hi = attn_hi(a, s, s.off + last / a.G);
    if (hi <= lo) return {0, 0};
    return {lo / kAttnStep, (hi + kAttnStep - 1) / kAttnStep - lo / kAttnStep};
}

// Workers that get a part: so few that each has two steps, four of tiles of 128 rows,
// about.  With all of them, however little that leaves each, a batch of few tiles spends
// its time on partial results: 32 tokens of 8 query heads to 2 key heads over 30000 keys
// 43 us against 36, of which 11 are the joining.
SQ_HD int attn_workers(const AttnShape& a, int64_t total) {
    const int64_t parts = divide(total, (int64_t)a.G * kAttnStep * (a.rows > 32 ? 4 : 2)) + 1;
    return parts < a.workers ? (int)parts : a.workers;
}
// The weight in equal parts: worker w's are positions [attn_start(w), attn_start(w + 1)).
struct AttnCut {
    int64_t each, more;           // the first `more` workers have one position more
};
SQ_HD AttnCut attn_cut_work(int64_t total, int workers) {
    const int64_t each = divide(total, workers);
    return {each, total - each * workers};
}
SQ_HD int64_t attn_start(const AttnCut& c, int w) { return w * c.each + (w < c.more ? w : c.more); }
// The worker whose part holds position x.
SQ_HD int attn_worker(const AttnCut& c, int64_t x) {
    const int64_t y = x - c.more * (c.each + 1);
    return (int)(y < 0 ? divide(x, c.each + 1) : c.more + divide(y, c.each));
}

// Of `count` steps of a tile of weight `weight`, those before fraction x / weight.
// 0 at 0 and count at weight, so the parts of a tile cover its steps once.
SQ_HD int attn_cut(int64_t x, int64_t weight, int count) {
    return x <= 0 ? 0 : x >= weight ? count : (int)divide(x * count + weight - 1, weight);
}

// What a worker that stands at position `at` and ends at `end` does of tile r of key
// head h: steps [k0, k1), where it stands next, whether these are all of the tile's
// (a tile without steps is its first worker's, which writes zeros), and whether its
// part begins and ends inside the tile.
struct AttnPart {
    int64_t next;
    int k0, k1;
    bool whole, begins_inside, ends_inside;
};
SQ_HD AttnPart attn_part(const AttnShape& a, const AttnSeq& q, int64_t before, int h, int r, int64_t at, int64_t end) {
    const int64_t weight = q.base + q.slope * r, from = before + h * q.weight + attn_before(q, r);
    const int64_t x0 = at - from, x1 = end - from < weight ? end - from : weight;
    const AttnSteps s = attn_steps(a, q.s, r);
    const int k0 = attn_cut(x0, weight, s.count), k1 = attn_cut(x1, weight, s.count);
    return {from + x1, s.first + k0, s.first + k1, k1 - k0 == s.count && (s.count > 0 || x0 == 0), x0 > 0, x1 < weight};
}

// The workspace of a batch whose tiles are shared out.  Every worker has two places for
// partial results: of the tile its part begins inside of, and of the one that begins in
// its part and ends in a later worker's.  Of the second it leaves the tile's last worker
// (-1: there is none) and a record: the joining kernel joins this worker's place for it
// and the first places of the workers up to the last.  A worker that has no step of a
// tile, or all of them and wrote the rows, leaves its place without a maximum (-inf).
// A first word says whether tiles are shared at all.
struct AttnRecord {
    int t0, rows;         // the sequence's first row of the batch, its rows of a key head
    int row0, h;          // the tile's first row and key head
};
SQ_HD int attn_place(int w, bool begins_inside) { return 2 * w + (begins_inside ? 0 : 1); }
// Per row of a tile: D sums in fp32, the reference and the sum of the row's softmax.
SQ_HD int64_t attn_place_floats(int rows, int D) { return (int64_t)rows * (D + 2); }
inline int64_t attn_workspace(const AttnShape& a, int D) {
    return 16 + a.workers * (4 + (int64_t)sizeof(AttnRecord) + 2 * attn_place_floats(a.rows, D) * 4);
}

// Tiles of all sequences and key heads, at most: places in a list where a batch is read
// tile by tile.
inline int64_t attn_tile_slots(const AttnShape& a) { return ((int64_t)a.T * a.G / a.rows + a.B) * a.heads; }

// Whether a batch is read with a workgroup for each tile instead, none split and
// nothing joined (direct).  `total` is all tiles' weight, `most` the largest tile's.
// Workgroups take tiles as they come free, so the last ends after about total / groups
// if no tile is longer than that; splitting saves at most most - total / groups, and
// costs the joining, as much as reading 1024 keys: one token over 518 keys 10.6 us
// against 17.5 split, 2048 tokens of one sequence 77 against 110; 32 tokens of lengths
// to 8192 55 us split.  (At 512 the first two split.  At 2048 tiles of 128 rows gain where
// there are about as many as workgroups, 3000 tokens of one sequence 165 -> 99 us, and lose
// for heads above 128, 1500 tokens 143 -> 236.)
// Decided by every workgroup, from the lengths, and all come to the same answer.
SQ_HD bool attn_always_direct(const AttnShape& a) { return a.max_len <= a.join; }   // all that the host can tell
SQ_HD bool attn_direct(const AttnShape& a, int64_t total, int64_t most) {
    return attn_always_direct(a) || most <= divide(total, a.groups) + (int64_t)a.G * a.join;
}

// Which kernel a call takes, by what the host knows: rows and the length that a page
// table row can hold, not the lengths themselves.
//   up to 16 rows a sequence and key head, on average: tiles of 16
//   up to 64: tiles of 32, of 16 for heads above 128
//   more: tiles of 128
// The first two read with single waves (four or eight of a workgroup, one workgroup a
// CU), the last with workgroups of four waves, two a CU.  Measured (us) with tiles of
// 16 / 32 / 128, 8 sequences of 32 heads of 128, 2000 older keys and another 12 tokens
// 28.4 / 33.2 / -, 24: 42.8 / 35.8 / 57.8, 56: 72.8 / 60.2 / 63.5, 96: - / 89.3 / 76.2,
// 128: - / 111.5 / 80.1.  Heads of 256 take 16 rows at a time, or 128 where there are
// more than 64 (4 x 1024 tokens 266 / - / 206).  A call has one size, by its average: 512
// tokens among 63 next tokens over caches of 2000 keys (32 heads to 32) take tiles of 16,
// 294 us, the two apart 63 and 217; with 8 key heads tiles of 32, 134 us, apart 64 and 55.
constexpr int kAttnCus = 256;

// Tiles of 128 rows read tile by tile: a head's tiles run on as few XCDs as share it,
// which read the same keys, and go round them one by one, so that each has its share of
// long sequences; the longest tiles of a sequence first.  Both together: 14 x 400 .. 862
// tokens over 4000 keys 583 -> 536 us, over 1000 225 -> 212; either alone gains less, and
// 8 prompts without older keys take the same time.
SQ_HD int attn_head_xcds(int heads) {
    const int low = heads & -heads;                     // 8 XCDs
    return low >= 8 ? 1 : 8 / low;
}
// Place `at` of a head's list, in which every XCD has a run of tiles / xcds: its tile.
SQ_HD int64_t attn_spread(int64_t at, int64_t tiles, int xcds) {
    const int64_t run = tiles / xcds;
    return at % run * xcds + at / run;
}

// Workgroups: a place for every tile, and those that share the work.
inline int64_t attn_grid(const AttnShape& a) {
    int64_t n = attn_tile_slots(a);
    if (!attn_always_direct(a) && n < a.groups) n = a.groups;
    const int64_t whole = a.heads * (a.rows > 32 ? attn_head_xcds(a.heads) : 1);
    return (n + whole - 1) / whole * whole;
}

// Waves of a workgroup that reads with single waves: what its registers hold without
// spilling (tiles of 32 of heads to 128: eight instead of four, 8 blocks of 32 tokens
// 39.0 -> 48.8 us).
inline int attn_waves(int rows, int D) { return rows * (D <= 64 ? 64 : D <= 128 ? 128 : 256) <= 16 * 128 ? 8 : 4; }

inline AttnShape attn_shape_of_rows(int rows, int T, int B, int Hq, int heads, int D, int max_len, bool causal,
                                    int window) {
    AttnShape a{T, B, heads, Hq / heads, max_len, causal, window, rows, kAttnCus, 0, 1024};
    if (rows == 128) a.groups = a.workers = D <= 128 ? 2 * kAttnCus : kAttnCus;
    else a.workers = a.groups * attn_waves(rows, D);
    return a;
}
inline AttnShape attn_shape(int T, int B, int Hq, int heads, int D, int max_len, bool causal, int window) {
    const int64_t rows = (int64_t)T * (Hq / heads);
    return attn_shape_of_rows(rows > (int64_t)64 * B ? 128 : rows > (int64_t)16 * B && D <= 128 ? 32 : 16, T, B, Hq,
                              heads, D, max_len, causal, window);
}

// The most that a batch of up to T tokens and B sequences needs: of every tile that one of
// them can take, so that a workspace made for the largest batch serves the others.
inline int64_t attn_workspace_most(int T, int B, int Hq, int heads, int D, int max_len) {
    const int64_t rows = (int64_t)T * (Hq / heads);
    int64_t most = 0;
    for (int r : {16, 32, 128}) {
        if ((r == 32 && (rows <= 16 || D > 128)) || (r == 128 && rows <= 64)) continue;
        const AttnShape a = attn_shape_of_rows(r, T, B, Hq, heads, D, max_len, true, 0);
        if (attn_always_direct(a)) return 0;
        const int64_t n = attn_workspace(a, D);
        most = n > most ? n : most;
    }
    return most;
}

}  // namespace sq
