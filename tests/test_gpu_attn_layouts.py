"""Head layouts at the ends of what is accepted: many query heads to a key head, so that a
token's rows are several tiles; many key heads; and a graph whose lengths change between
replays, so that the same captured kernels read whole tiles and shared ones."""
import numpy as np
import pytest
import torch

import paper_2606_04945_amd as sq
from attn_cases import check_attention, filled_cache, normal, ragged, to_device
from gpu_util import dev, host
from oracle import attn as A

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page,heads,G,dim,news,lens", [
    (32, 1, 300, 16, [1, 2], [90, 40]),                  # several tiles of 128 to a token
    (64, 1, 1024, 32, [1], [130]),
    (16, 1, 40, 256, [1], [1500]),
    (16, 700, 1, 16, [1, 2], [33, 20]),
    (64, 1024, 1, 32, [1], [70]),
    (128, 341, 3, 16, [3], [140]),
])
@pytest.mark.parametrize("window", [0, 25])
def test_heads(page, heads, G, dim, news, lens, window):
    rng = np.random.default_rng(heads + G)
    pages = sum(-(-L // page) for L in lens) + 1
    cu, ln, table = ragged(news, lens, max(-(-L // page) for L in lens), page, pages, rng)
    c = filled_cache(pages, heads, dim, page, rng)
    q = normal(rng, sum(news), heads * G, dim)
    for causal in (True, False):
        out, lse = sq.attn_kv8(dev(q), to_device(c), dev(cu), dev(ln), dev(table), causal=causal, window=window,
                               want_lse=True)
        check_attention(out, A.attention(q, c, cu, ln, table, causal, window), (causal, window), lse)


@pytest.mark.parametrize("G,dim,n", [(4, 128, 2), (1, 64, 40), (2, 128, 70)])
def test_lengths_change_between_replays(G, dim, n):
    rng = np.random.default_rng(dim)
    page, heads, B, room = 64, 2, 2, 45
    pages = 2 * room
    c = filled_cache(pages, heads, dim, page, rng)
    table = rng.permutation(pages).astype(np.int32).reshape(B, room)
    cu = np.array([0, n, 2 * n], np.int32)
    q = normal(rng, 2 * n, heads * G, dim)
    cache, d_q, d_cu, d_ln, d_t = to_device(c), dev(q), dev(cu), dev(np.array([n, n], np.int32)), dev(table)
    args = (d_q, cache, d_cu, d_ln, d_t)
    out, lse = sq.attn_kv8(*args, want_lse=True)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sq.attn_kv8(*args, out=out, lse=lse)
    for lens in ([n, n + 5], [2800, n], [200, 300], [0, 2700], [2880, 2880], [100, 100]):
        ln = np.array(lens, np.int32)
        d_ln.copy_(dev(ln))
        out.fill_(9), lse.fill_(9)
        g.replay()
        ref = A.attention(q, c, cu, ln, table)
        check_attention(out, ref, lens, lse)
        eager = sq.attn_kv8(*args, want_lse=True)
        assert torch.equal(eager[0], out) and torch.equal(eager[1], lse)
