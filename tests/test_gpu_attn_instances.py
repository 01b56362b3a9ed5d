"""Every instance of the attention kernels against the oracle (test_attn_instances_plan.py
says that these are all), each with and without a causal mask and with windows."""
import numpy as np
import pytest
import torch

import paper_2606_04945_amd as sq
from attn_cases import check_attention, filled_cache, normal, ragged, strided, to_device
from attn_instances import CASES, MASKS
from gpu_util import dev, host
from oracle import attn as A

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page,heads,G,dim,news,lens", CASES)
def test_instance(page, heads, G, dim, news, lens):
    rng = np.random.default_rng(page + dim + sum(news))
    pages = sum(-(-L // page) for L in lens) + 2
    cu, ln, table = ragged(news, lens, max(-(-L // page) for L in lens), page, pages, rng)
    c = filled_cache(pages, heads, dim, page, rng)
    q = normal(rng, sum(news) + 1, heads * G, dim)
    cache, table[-1, 0] = to_device(c), -1                # the last sequence's first page is none
    args = (strided(q), cache, dev(cu), dev(ln), dev(table))
    for causal, window in MASKS:
        out = torch.full(q.shape, 9.0, dtype=torch.float16, device="cuda")
        lse = torch.full(q.shape[:2], 9.0, dtype=torch.float32, device="cuda")
        sq.attn_kv8(*args, causal=causal, window=window, out=out, lse=lse)
        check_attention(out, A.attention(q, c, cu, ln, table, causal, window), (causal, window), lse)
        assert (host(out)[-1] == 9).all() and (host(lse)[-1] == 9).all()
