"""Attention over the block-scaled FP8 KV cache at the ends of its numbers' range, in tiles of 16 and of 128 rows, whole
and cut into runs: values up to the largest that the cache holds, scores up to the largest that fp32 holds."""
import numpy as np
import pytest
import torch

import kvb_plain as P
import paper_2606_20537_amd as cap
from test_gpu_kvb import BLOCK, Caches, append, check_attend, normal, reread, run_attend, up

pytestmark = pytest.mark.gpu

# rows held, tokens, query heads on one KV head, copies in one call: tiles of 16, whole and in runs; of 128,
# whole and in runs
NARROW = [(500, 5, 3, 1), (3000, 1, 8, 1)]
WIDE = [(1100, 90, 8, 32), (4500, 161, 16, 1)]


def made(n, d, k, v, fill=0x7F):
    c = Caches([up(n)], 1, d, fill)
    append(c, [0], [n], [k], [v])
    return c, *reread(c, [n])


def rising(n, d, by):
    """Keys whose product with a query of (1, 0, ...) rises by `by` from the first block to the second, then stays."""
    k = torch.zeros(n, 1, d)
    k[:, 0, 0] = by
    k[:BLOCK, 0, 0] = 0.0
    return k.bfloat16()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n, T, G, copies", NARROW + WIDE)
@pytest.mark.parametrize("size, by", [(2.0 ** 70, 40.0), (2.0 ** 70, -40.0), (2.0 ** 121, 0.0), (2.0 ** 121, 40.0), (3.3e38, 0.0), (3.3e38, -0.5)])
def test_large_values(d, n, T, G, copies, size, by):
    """Means of values up to the largest stay finite, whatever the scores before them were."""
    v = normal(1, n, 1, d).float().clamp(-1, 1) * size
    if size > 1e38:
        v = v.abs().clamp(size / 2)  # sums far beyond the type's largest number
    c, ks, vs = made(n, d, rising(n, d, by), v.bfloat16())
    q = torch.zeros(T, G, d).bfloat16().cuda()
    q[..., 0] = 1.0
    o, lse = run_attend(c, [n], [T], q, 1.0, copies=copies)
    assert torch.isfinite(o).all()
    check_attend(c, ks, vs, [n], [T], q, 1.0, o, lse, rows=100)


@pytest.mark.parametrize("d", [64, 256])
@pytest.mark.parametrize("size", [2.0 ** 96, 3.3e38])
def test_large_values_of_listed_blocks(d, size):
    """The same over block lists, with repetitions and a token that sees nothing."""
    n, T, G = 2000, 3, 8
    v = normal(5, n, 1, d).float().abs().clamp(0.5, 1) * size
    c, ks, vs = made(n, d, rising(n, d, 1.0), v.bfloat16())
    q = torch.ones(T, G, d).bfloat16().cuda()
    idx = (torch.arange(T * 100, dtype=torch.int32) % 31).view(T, 1, 100).cuda()
    idx[1] = -1
    o, lse = run_attend(c, [n], [T], q, 1.0, idx)
    assert torch.isfinite(o).all() and not o[1].any()
    check_attend(c, ks, vs, [n], [T], q, 1.0, o, lse, idx)
