"""Work division of the attention over the cache, on the CPU: the package's planning
code compiled with g++, every worker and every joining workgroup walked as the kernels
walk them."""
import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_04945_amd", "csrc")
SHIM = r"""
#include <map>
#include <set>
#include <tuple>
#include <vector>
#include "attn_plan.hpp"
using namespace sq;

// 0 if every step of every tile is read once, every split tile is joined from exactly the places written for
// it, and every index stays inside its bounds; otherwise a number that says what was wrong.
extern "C" int walk(int T, int B, int heads, int G, int max_len, int causal, int window, int rows, int at_once,
                    const int* cu, const int* lens, long long* stats) {
    const AttnShape a{T, B, heads, G, max_len, causal, window, rows, at_once, at_once, 0};
    std::vector<AttnSeq> s;
    std::vector<int64_t> before;
    int64_t total = 0;
    for (int b = 0; b < B; ++b) {
        s.push_back(attn_seq(a, cu[b], cu[b + 1], lens[b]));
        if (s[b].s.t0 < 0 || s[b].s.t0 + s[b].s.n > T || s[b].s.n < 0 || s[b].s.len < 0 || s[b].s.len > max_len) return 2;
        if (s[b].weight < 0 || (s[b].weight == 0) != (s[b].s.n == 0)) return 3;
        before.push_back(total);
        total += s[b].weight * heads;
    }
    typedef std::tuple<int, int, int> Tile;
    std::map<Tile, std::vector<int>> read;                 // how often each step is read
    std::map<Tile, std::map<int, bool>> written;           // places: whether they hold a result
    std::map<Tile, int> direct;
    std::set<int> places;
    std::vector<int> lasts(a.workers, -1);
    const int workers = attn_workers(a, total);
    if (workers < 1 || workers > a.workers) return 24;
    std::vector<Tile> recorded(a.workers);
    int64_t most = 0, least = INT64_MAX;
    const AttnCut cut = attn_cut_work(total, workers);
    if (attn_start(cut, 0) != 0 || attn_start(cut, workers) != total) return 16;
    for (int w = 0; w < workers; ++w) {
        int64_t at = attn_start(cut, w), end = attn_start(cut, w + 1), did = 0;
        if (end < at) return 4;
        int b = 0;
        while (at < end) {
            if (b >= B) return 5;
            const AttnSeq& q = s[b];
            if (at - before[b] >= q.weight * heads) { ++b; continue; }
            const int h = (int)divide(at - before[b], q.weight);
            if (h < 0 || h >= heads) return 6;
            const int r = attn_find_tile(q, at - before[b] - h * q.weight);
            const int64_t weight = q.base + q.slope * r, from = before[b] + h * q.weight + attn_before(q, r);
            if (at < from || at >= from + weight) return 7;
            const AttnPart part = attn_part(a, q, before[b], h, r, at, end);
            if (part.next <= at || part.next > end || part.next > from + weight) return 7;
            if (part.begins_inside != (at > from) || part.ends_inside != (part.next < from + weight)) return 18;
            const Tile t(b, h, r);
            if (part.ends_inside && !part.begins_inside) {
                if (lasts[w] >= 0) return 19;
                lasts[w] = attn_worker(cut, from + weight - 1);
                recorded[w] = t;
                if (lasts[w] <= w || lasts[w] >= workers) return 20;
            }
            at = part.next;
            const AttnSteps st = attn_steps(a, q.s, r);
            if (st.count < 0 || st.first < 0 || (st.count && (int64_t)(st.first + st.count - 1) * kAttnStep >= q.s.len)) return 8;
            if (part.k0 < st.first || part.k1 > st.first + st.count || part.k1 < part.k0) return 17;
            read[t].resize(st.count);
            for (int k = part.k0; k < part.k1; ++k) ++read[t][k - st.first];
            did += part.k1 - part.k0;
            direct[t] += part.whole;
            if (part.begins_inside || part.ends_inside) {
                const int place = attn_place(w, part.begins_inside);
                if (place < 0 || place >= 2 * a.workers || !places.insert(place).second) return 9;
                written[t][place] = part.k0 < part.k1 && !part.whole;
            } else if (!part.whole) return 21;
        }
        if (attn_start(cut, w) >= end) continue;
        most = std::max(most, did);
        least = std::min(least, did);
    }
    int64_t slots = attn_tile_slots(a);
    std::map<Tile, int> joined;
    for (int w = 0; w < workers; ++w)
        if (lasts[w] >= 0) {
            std::map<int, bool> join;
            for (int j = w; j <= lasts[w]; ++j) {
                const int place = attn_place(j, j > w);
                if (!written[recorded[w]].count(place)) return 22;
                join[place] = written[recorded[w]][place];
            }
            if (join != written[recorded[w]]) return 23;
            ++joined[recorded[w]];
        }
    long long split = 0;
    for (int b = 0; b < B; ++b) {
        const AttnSeq& q = s[b];
        for (int h = 0; h < heads; ++h)
            for (int r = 0; r < q.tiles; ++r) {
                Tile t(b, h, r);
                const AttnSteps st = attn_steps(a, q.s, r);
                const auto& c = read[t];
                if ((int)c.size() != st.count) return 10;
                for (int x : c) if (x != 1) return 11;
                // the steps hold every visible key of every row of the tile
                for (int64_t row = (int64_t)r * rows; row < std::min<int64_t>((int64_t)(r + 1) * rows, (int64_t)q.s.n * G); ++row) {
                    const int p = q.s.off + (int)(row / G), lo = attn_lo(a, p), hi = attn_hi(a, q.s, p);
                    if (hi > lo && (lo < st.first * kAttnStep || hi > (st.first + st.count) * kAttnStep)) return 12;
                }
                // a batch read tile by tile finds every tile
                const int64_t item = list_start(q.s.t0, b, G, rows, 1) + r;
                if (item * heads + h >= slots) return 13;
                int lo = -1;
                for (int i = 0; i < B; ++i) lo += list_start(std::min(std::max(cu[i], 0), T), i, G, rows, 1) <= item;
                if (lo != b) return 14;
                // written by one worker, or joined from results, once
                bool any = false;
                for (auto& x : written[t]) any |= x.second;
                if (direct[t] != !any || joined[t] != !written[t].empty()) return 15;
                split += any;
            }
    }
    stats[0] = most; stats[1] = least; stats[2] = split; stats[3] = a.workers;
    return 0;
}

extern "C" int plan(int T, int B, int Hq, int heads, int D, int max_len, int* o) {
    const AttnShape a = attn_shape(T, B, Hq, heads, D, max_len, true, 0);
    o[0] = a.groups; o[1] = a.workers; o[2] = attn_always_direct(a);
    if (attn_grid(a) < attn_tile_slots(a) || (!o[2] && attn_grid(a) < a.groups)) return 0;
    return a.rows;
}

// 0 if the grid of tiles of 128 rows read tile by tile has every tile of every head once, and how far the XCDs'
// numbers of places lie apart.
extern "C" int spread(int T, int B, int heads, int G, int* apart) {
    AttnShape a = attn_shape(T, B, heads * G, heads, 128, 1 << 20, true, 0);
    a.rows = 128;
    const int64_t grid = attn_grid(a), tiles = grid / heads;
    if (grid % heads || tiles % attn_head_xcds(heads) || grid < attn_tile_slots(a)) return 1;
    std::set<int64_t> seen;
    for (int64_t at = 0; at < tiles; ++at) {
        const int64_t t = attn_spread(at, tiles, attn_head_xcds(heads));
        if (t < 0 || t >= tiles || !seen.insert(t).second) return 2;
    }
    *apart = (int)(grid % 8);
    return 0;
}

// Whether a step of every sequence, `heads` key heads of G query heads, is read without splitting.
extern "C" int direct(int B, int heads, int G, int max_len, int n, const int* lens) {
    const AttnShape a = attn_shape(B * n, B, heads * G, heads, 128, max_len, true, 0);
    int64_t total = 0, most = 0;
    for (int b = 0; b < B; ++b) {
        const AttnSeq q = attn_seq(a, b * n, b * n + n, lens[b]);
        total += q.weight * heads;
        most = std::max(most, q.base + q.slope * (q.tiles - 1));
    }
    return attn_direct(a, total, most);
}

extern "C" int touched(int T, int B, int max_len, int page, const int* cu, const int* lens) {
    std::set<std::pair<int64_t, int>> seen;
    for (int b = 0; b < B; ++b) {
        const Seq s = make_seq(cu[b], cu[b + 1], lens[b], T, max_len);
        const int n = touched_count(s, page);
        for (int j = 0; j < n; ++j) {
            const int64_t item = list_start(s.t0, b, 1, page, 2) + j;
            if (item < 0 || item >= touched_slots(T, B, page)) return 1;
            int lo = 0, hi = B - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) / 2, cm = std::min(std::max(cu[mid], 0), T);
                if (list_start(cm, mid, 1, page, 2) <= item) lo = mid; else hi = mid - 1;
            }
            if (lo != b) return 2;
            const int blk = touched_first(s, page) + j;
            if (blk * (int64_t)page >= max_len || blk < 0) return 3;
            if (std::max(s.off, blk * page) >= std::min(s.len, (blk + 1) * page)) return 4;
        }
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("attn_plan")
    (d / "shim.cpp").write_text("#include <algorithm>\n" + SHIM)
    so = str(d / "shim.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(d / "shim.cpp"), "-o", so],
                   check=True)
    return ctypes.CDLL(so)


def ints(v):
    return (ctypes.c_int * len(v))(*v)


def walk(plan, T, B, heads, G, max_len, causal, window, rows, at_once, cu, lens):
    stats = (ctypes.c_longlong * 4)()
    rc = plan.walk(T, B, heads, G, max_len, causal, window, rows, at_once, ints(cu), ints(lens), stats)
    return rc, list(stats)


def batch(rng, most_new, most_old, B):
    cu, lens = [0], []
    for _ in range(B):
        n = rng.choice([0, 1, 1, rng.randint(0, most_new)])
        cu.append(cu[-1] + n)
        lens.append(max(0, rng.choice([n, n + rng.randint(0, most_old), rng.randint(0, most_old)])))
    return cu, lens


@pytest.mark.parametrize("seed", range(300))
def test_every_step_once(plan, seed):
    rng = random.Random(seed)
    B = rng.choice([1, 1, 2, 7, 70])
    cu, lens = batch(rng, rng.choice([1, 5, 200]), rng.choice([3, 200, 3000]), B)
    T = cu[-1] + rng.randint(0, 4)
    max_len = max(lens) + rng.choice([0, 1, 100, 10000])
    rc, _ = walk(plan, T, B, rng.choice([1, 2, 8]), rng.choice([1, 3, 7, 20]), max_len, rng.randint(0, 1),
                 rng.choice([0, 0, 1, 50, 700]), rng.choice([16, 64, 128]), rng.choice([1, 8, 512, 2048]), cu, lens)
    assert rc == 0


@pytest.mark.parametrize("seed", range(100))
def test_any_index_values_stay_inside(plan, seed):
    """Rows, lengths of any value: nothing outside the bounds (a tile then may be read by nobody or twice)."""
    rng = random.Random(1000 + seed)
    B = rng.choice([1, 3, 9])
    wild = [-2 ** 31, -1, 0, 3, 17, 1000, 2 ** 31 - 1]
    cu = [rng.choice(wild) for _ in range(B + 1)]
    lens = [rng.choice(wild) for _ in range(B)]
    rc, _ = walk(plan, 20, B, 2, 3, 500, seed % 2, rng.choice([0, 9]), 16, 64, cu, lens)
    assert rc in (0, 10, 11, 13, 14, 15)
    assert plan.touched(20, B, 500, 16, ints(cu), ints(lens)) in (0, 1, 2)


@pytest.mark.parametrize("seed", range(200))
def test_every_touched_page_has_a_place(plan, seed):
    rng = random.Random(seed)
    B = rng.choice([1, 2, 7, 70])
    cu, lens = batch(rng, rng.choice([1, 5, 300]), rng.choice([3, 200, 3000]), B)
    assert plan.touched(cu[-1], B, max(lens) + 64, rng.choice([16, 32, 64, 128]), ints(cu), ints(lens)) == 0


def test_load_is_even(plan):
    """One long sequence among short ones: no worker reads more than its share and a step or two."""
    lens = [100000] + [50] * 31
    rc, (most, least, split, workers) = walk(plan, 32, 32, 8, 7, 131072, 1, 0, 16, 2048, list(range(33)), lens)
    steps = 8 * sum(-(-L // 64) for L in lens)
    assert rc == 0 and workers == 2048 and split == 8
    assert most <= steps / workers + 3


def test_largest_sizes_do_not_overflow(plan):
    """Weights stay in 64 bits at the limits the interface accepts."""
    T, heads, G, max_len = 1 << 20, 1, 16, 1 << 28
    rc, _ = walk(plan, T, 1, heads, G, max_len, 1, 0, 128, 4, [0, 1 << 10], [max_len])
    assert rc == 0


def test_which_kernel(plan):
    """Rows a tile, workgroups, workers and whether nothing can be split, by rows, heads and room of the page table."""
    def shape(*a):
        o = (ctypes.c_int * 3)()
        return plan.plan(*a, o), *o
    assert shape(1, 1, 32, 32, 128, 512) == (16, 256, 2048, 1)
    assert shape(32, 32, 28, 4, 128, 8192) == (16, 256, 2048, 0)
    assert shape(2, 2, 64, 8, 256, 131072) == (16, 256, 1024, 0)
    assert shape(8 * 32, 8, 32, 32, 128, 2112) == (32, 256, 1024, 0)
    assert shape(8 * 32, 8, 32, 32, 64, 320) == (32, 256, 2048, 1)
    assert shape(8 * 2048, 8, 28, 4, 128, 2048) == (128, 512, 512, 0)
    assert shape(32, 1, 28, 4, 256, 64) == (128, 256, 256, 1)


def test_tiles_go_round_the_xcds(plan):
    for seed in range(60):
        rng = random.Random(seed)
        apart = ctypes.c_int(-1)
        B = rng.randint(1, 40)
        assert plan.spread(rng.randint(B, 5000), B, rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 12, 16, 28, 32]),
                           rng.randint(1, 16), ctypes.byref(apart)) == 0
        assert apart.value == 0


def test_direct_or_shared(plan):
    """Tile by tile where no tile is much longer than a workgroup's share, or the difference is small."""
    def direct(lens, heads, G, n=1, room=1 << 20):
        return plan.direct(len(lens), heads, G, room, n, ints(lens))
    assert direct([517], 32, 1)                               # short
    assert not direct([131072] * 2, 8, 8)                     # 16 tiles of 256 workgroups'
    assert direct([2000] * 8, 32, 1, 32)                      # a tile a workgroup, even
    assert not direct([100000] + [100] * 63, 8, 4)            # one long sequence
    assert direct([3000] * 256, 4, 7) and direct([1500] * 8, 4, 7, 1500)
    for seed in range(50):                                    # a narrow table: whatever the lengths
        rng = random.Random(seed)
        assert direct([rng.randint(0, 1024) for _ in range(rng.randint(1, 9))], 2, 4, rng.choice([1, 40]), 1024)
