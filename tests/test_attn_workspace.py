"""The attention's workspace on the CPU: one made for the largest batch serves smaller ones."""
import random

import pytest

from paper_2606_04945_amd import _lib as L
from test_attn_plan import plan  # noqa: F401  (the plan compiled with g++)


@pytest.fixture(scope="module")
def need():
    return L.lib().sq_attn_kv8_workspace_bytes


@pytest.mark.parametrize("heads,G,dim", [(8, 1, 64), (8, 1, 128), (4, 7, 128), (2, 20, 96), (1, 8, 256), (2, 1, 16)])
def test_never_less_for_more(need, heads, G, dim):
    rng = random.Random(dim + G)
    for B in (1, 2, 16, 300):
        sizes = sorted({1, 2, 3, 9, 16, 17, 33, 64, 65, 129, 511, 512, 513, 1024, 1025, 1088, 2048, 5000, B, 16 * B,
                        16 * B + 1, 64 * B, 64 * B + 1, *(rng.randint(1, 20000) for _ in range(50))})
        for max_len in (1024, 1040, 8192):
            got = [need(T, B, heads * G, heads, dim, max_len) for T in sizes]
            assert got == sorted(got), (B, max_len)
            assert got[-1] >= need(sizes[-1], max(1, B // 2), heads * G, heads, dim, max_len)
            for T, n in zip(sizes, got):
                assert n >= need(rng.randint(1, T), rng.randint(1, B), heads * G, heads, dim, max_len)
                assert n >= need(T, B, heads * G, heads, dim, max_len // 2)


def test_what_a_call_uses_fits(need, plan):  # noqa: F811
    """Rows and workers that the plan takes, two places of partial results a worker."""
    import ctypes
    rng = random.Random(1)
    for _ in range(300):
        heads, G, dim = rng.choice([(8, 1, 64), (4, 7, 128), (2, 20, 96), (1, 8, 256)])
        T, B, room = rng.randint(1, 3000), rng.randint(1, 100), rng.choice([512, 2048, 100000])
        o = (ctypes.c_int * 3)()
        rows = plan.plan(T, B, heads * G, heads, dim, room, o)
        used = 0 if o[2] else 16 + o[1] * (4 + 16 + 2 * rows * (dim + 2) * 4)
        n = need(T, B, heads * G, heads, dim, room)
        assert n >= used and (n == 0) == (used == 0)
