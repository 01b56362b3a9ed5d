"""Which instance of the attention kernels each of the tested batches takes, asked of the
planning code compiled with g++: every one has a case, with and without a causal mask and a
window."""
import ctypes
import os
import subprocess

import pytest

from attn_instances import CASES, MASKS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_04945_amd", "csrc")
SHIM = r"""
#include <algorithm>
#include "attn_plan.hpp"
using namespace sq;

// o: rows a tile, whether a workgroup has a whole tile, and of shared batches how many tiles are split
extern "C" void instance(int T, int B, int heads, int G, int D, int max_len, int causal, int window, const int* cu,
                         const int* lens, int* o) {
    const AttnShape a = attn_shape(T, B, heads * G, heads, D, max_len, causal, window);
    int64_t total = 0, most = 0;
    for (int b = 0; b < B; ++b) {
        const AttnSeq q = attn_seq(a, cu[b], cu[b + 1], lens[b]);
        total += q.weight * heads;
        most = std::max(most, attn_most(q));
    }
    o[0] = a.rows;
    o[1] = attn_direct(a, total, most);
    o[2] = 0;
    if (o[1]) return;
    const int workers = attn_workers(a, total);
    const AttnCut cut = attn_cut_work(total, workers);
    int64_t before = 0;
    for (int b = 0; b < B; ++b) {
        const AttnSeq q = attn_seq(a, cu[b], cu[b + 1], lens[b]);
        for (int h = 0; h < heads; ++h)
            for (int r = 0; r < q.tiles; ++r) {
                const int64_t from = before + h * q.weight + attn_before(q, r), w = q.base + q.slope * r;
                o[2] += attn_worker(cut, from) != attn_worker(cut, from + w - 1);
            }
        before += q.weight * heads;
    }
}
"""


@pytest.fixture(scope="module")
def instance(tmp_path_factory):
    d = tmp_path_factory.mktemp("attn_instances")
    (d / "shim.cpp").write_text(SHIM)
    so = str(d / "shim.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(d / "shim.cpp"), "-o", so],
                   check=True)
    lib = ctypes.CDLL(so)

    def ask(page, heads, G, dim, news, lens, causal, window):
        cu = [sum(news[:b]) for b in range(len(news) + 1)]
        ints = lambda v: (ctypes.c_int * len(v))(*v)  # noqa: E731
        o = (ctypes.c_int * 3)()
        room = max(-(-L // page) for L in lens) * page
        lib.instance(sum(news), len(news), heads, G, dim, room, int(causal), window, ints(cu), ints(lens), o)
        return o[0], 64 if dim <= 64 else 128 if dim <= 128 else 256, page >= 64, bool(o[1]), o[2]
    return ask


def test_every_instance_is_tested(instance):
    want = {(rows, heads, wide, direct) for rows, sizes in ((16, (64, 128, 256)), (32, (64, 128)), (128, (64, 128, 256)))
            for heads in sizes for wide in (False, True) for direct in (False, True)}
    for causal, window in MASKS[:3]:
        got = {i[:4] for i in (instance(*c, causal, window) for c in CASES) if i[3] or i[4]}
        assert got == want, (causal, window, want - got)
    for causal, window in MASKS[3:]:                      # short windows leave nothing to share
        assert {i[:3] for i in (instance(*c, causal, window) for c in CASES)} == {w[:3] for w in want}


def test_every_head_size_is_tested_somewhere():
    assert {d for _, _, _, d, _, _ in CASES} >= {16, 64, 80, 96, 112, 128, 144, 160, 192, 208, 256}
