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
LONG = (8400, 70, 32, 48)  # tiles of 128, more than 128 blocks in a run


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


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n, T, G, copies", NARROW + WIDE)
@pytest.mark.parametrize("by", [-80.0, -84.0, -87.0, -120.0, -1000.0])
@pytest.mark.parametrize("parts", [(0, 64), (32, 96), (0, 32)])
def test_large_values_of_keys_far_below(d, n, T, G, copies, by, parts):
    """The largest values at keys whose scores are so far below the others' that nothing of them is left (or, 2^115 below,
    a tenth of the others), whether they fill a block, halves of two blocks, or half of one."""
    k, v = torch.zeros(n, 1, d), normal(6, n, 1, d).float()
    for b in range(0, n, 3 * BLOCK):
        k[b + parts[0]:b + parts[1], 0, 0] = by
        v[b + parts[0]:b + parts[1]] = 2.0 ** 115
    c, ks, vs = made(n, d, k.bfloat16(), v.bfloat16())
    q = torch.zeros(T, G, d).bfloat16().cuda()
    q[..., 0] = 1.0
    o, lse = run_attend(c, [n], [T], q, 1.0, copies=copies)
    for t, h in [(t, h) for t in (0, T // 2, T - 1) for h in (0, G - 1)]:
        row, pos = q[t, h].double().cpu().numpy(), n - T + t
        want, want_lse, mass, top, size = P.attend(row, ks[0][:, 0], vs[0][:, 0], 1.0, pos)
        # as kvb_plain.close has it, and weights below 2^-80 of the largest may count as none
        x = ks[0][:pos + 1, 0] @ row
        weight = np.exp(x - want_lse)
        none = (weight * (weight < weight.max() * 2.0 ** -80)) @ np.abs(vs[0][:pos + 1, 0])
        far = mass * (2.0 ** -8 + 2 * (d * 2.0 ** -24 * size + 2.0 ** -22 * (abs(want_lse) + size))) + 1e-37 + none
        if T * G > 128:
            # lo's step is 2^-21 of the block's largest weight at most: a weight below half of it is lost, no more
            block = np.arange(pos + 1) // BLOCK
            largest = np.array([weight[block == b].max() for b in range(block[-1] + 1)])[block]
            far = far + mass * 2.0 ** -12 + np.minimum(weight, 2.0 ** -21 * largest) @ np.abs(vs[0][:pos + 1, 0])
        far = far + 2.0 ** -8 * (np.abs(want) + far)
        got = o[t, h].double().cpu().numpy()
        assert (np.abs(got - want) <= far).all(), (t, h, np.abs(got - want).max(), far.min(), np.abs(want).max())
        assert abs(lse[t, h].item() - want_lse) <= 2.0 ** -20 * (1 + abs(want_lse))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n, T, G, copies", NARROW + WIDE)
@pytest.mark.parametrize("scale", [3e4, -3e4, 1e6, -1e6, 1e20, -1e20])
def test_large_scores(d, n, T, G, copies, scale):
    """Scores far above 2^24, whose roundings are larger than one: the mean of the keys with the highest score, from the
    first blocks to the last, whichever score that is.  Products of q and k are integers, so that equal scores are equal in
    any arithmetic and others lie `scale` apart at least."""
    g = torch.Generator().manual_seed(8)
    k, q = (torch.randint(-3, 4, shape, generator=g).float() for shape in ((n, 1, d), (T, G, d)))
    k, q = k * 8, q * 8  # (products of 64 and more: scores above 2^24 from a scale of 3e4 on)
    c, ks, vs = made(n, d, k.bfloat16(), normal(9, n, 1, d))
    o, lse = run_attend(c, [n], [T], q.bfloat16().cuda(), scale, copies=copies)
    scale = float(np.float32(scale))
    for t, h in {(t, h) for t in range(0, T, max(1, T // 40)) for h in (0, G // 2, G - 1)}:
        pos = n - T + t
        x = (ks[0][:pos + 1, 0] @ q[t, h].double().numpy()) * np.sign(scale)
        best = vs[0][:pos + 1, 0][x == x.max()]
        want, mass, want_lse = best.mean(0), np.abs(best).mean(0), abs(scale) * x.max() + np.log(len(best))
        # equal weights are rounded alike, the sum of 64 products by 2^-12 of their magnitudes, the output by 2^-8; the
        # other weights are no higher than 2^-126 of the sum: up to 2^8 times the instruction's smallest scale 2^-127 (and
        # their low halves, up to 2^3, times the same), against 2^7 and more
        far = mass * 2.0 ** -12 + 2.0 ** -125 * np.abs(vs[0][:pos + 1, 0]).sum(0)
        far = far + 2.0 ** -8 * (np.abs(want) + far)
        got = o[t, h].double().cpu().numpy()
        assert (np.abs(got - want) <= far).all(), (t, h, len(best), np.abs(got - want).max())
        # scale log2(e), its product with the score and the way back are each rounded
        assert abs(lse[t, h].item() - want_lse) <= 2.0 ** -21 * abs(want_lse)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n, T, G, copies", NARROW + WIDE)
@pytest.mark.parametrize("q_size, k_size, scale", [(2.0 ** 124, 2.0 ** -93, 2.0 ** -34), (2.0 ** -118, 2.0 ** 120, 2.0 ** -5), (2.0 ** -90, 2.0 ** -20, 2.0 ** 107)])
def test_queries_and_keys_of_unlike_sizes(d, n, T, G, copies, q_size, k_size, scale):
    """Queries and keys at opposite ends of the range, with scores of ordinary size."""
    k, q = normal(10, n, 1, d).float().clamp(-4, 4) * k_size, normal(11, T, G, d).float().clamp(-4, 4) * q_size
    c, ks, vs = made(n, d, k.bfloat16(), normal(12, n, 1, d))
    q = q.bfloat16().cuda()
    o, lse = run_attend(c, [n], [T], q, scale, copies=copies)
    check_attend(c, ks, vs, [n], [T], q, scale, o, lse, rows=100)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_long_runs(d):
    """Runs of more than 128 blocks, whose scales are loaded 64 blocks at a time: sizes of K and V that differ from block
    to block."""
    n, T, G, copies = LONG
    by = 2.0 ** torch.randint(-6, 7, (up(n) // BLOCK, 2), generator=torch.Generator().manual_seed(13)).float().repeat_interleave(BLOCK, 0)[:n]
    c, ks, vs = made(n, d, (normal(14, n, 1, d).float() * by[:, :1, None]).bfloat16(), (normal(15, n, 1, d).float() * by[:, 1:, None]).bfloat16())
    q = normal(16, T, G, d).cuda()
    o, lse = run_attend(c, [n], [T], q, 0.02, copies=copies)
    check_attend(c, ks, vs, [n], [T], q, 0.02, o, lse, rows=60)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("block", [0, 63, 64, 66, 127, 130])
def test_large_scores_of_one_block(d, block):
    """Scores above 2^24 in one block of a long run alone: the mean of that block's best keys, and of the others' rows
    that do not see it what they see."""
    n, T, G, copies = LONG
    g = torch.Generator().manual_seed(17)
    k, q = torch.zeros(n, 1, d), torch.full((T, G, d), 8.0)
    rows = k[block * BLOCK:(block + 1) * BLOCK]
    rows[:] = 8.0 * torch.randint(0, 3, rows.shape, generator=g)
    c, ks, vs = made(n, d, k.bfloat16(), normal(18, n, 1, d))
    o, lse = run_attend(c, [n], [T], q.bfloat16().cuda(), 1e6, copies=copies)
    for t in (0, T - 1):
        pos = n - T + t
        x = ks[0][:pos + 1, 0] @ q[t, 0].double().numpy()
        best = vs[0][:pos + 1, 0][x == x.max()]
        want, mass = best.mean(0), np.abs(best).mean(0)
        far = mass * 2.0 ** -12 + 2.0 ** -125 * np.abs(vs[0][:pos + 1, 0]).sum(0)  # as in test_large_scores
        far = far + 2.0 ** -8 * (np.abs(want) + far)
        for h in (0, G - 1):
            got = o[t, h].double().cpu().numpy()
            assert (np.abs(got - want) <= far).all(), (t, h, len(best), np.abs(got - want).max())
            assert abs(lse[t, h].item() - (1e6 * x.max() + np.log(len(best)))) <= 2.0 ** -21 * 1e6 * x.max() + 2.0 ** -20


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n_sel", [3, 8, 31, 90])
def test_sizes_that_differ_by_block_in_lists(d, n_sel):
    """Each listed block with scales of its own, in lists of one run and of several, with holes, blocks behind the token and
    repetitions: a block's codes never meet another's scale."""
    n, T, G = 2500, 4, 8
    by = 2.0 ** torch.randint(-8, 3, (up(n) // BLOCK, 2), generator=torch.Generator().manual_seed(19)).float().repeat_interleave(BLOCK, 0)[:n]
    c, ks, vs = made(n, d, (normal(20, n, 1, d).float() * by[:, :1, None]).bfloat16(), (normal(21, n, 1, d).float() * by[:, 1:, None]).bfloat16())
    q = normal(22, T, G, d).cuda()
    idx = torch.randint(-1, 42, (T, 1, n_sel), generator=torch.Generator().manual_seed(n_sel), dtype=torch.int32).cuda()
    o, lse = run_attend(c, [n], [T], q, 0.05, idx)
    check_attend(c, ks, vs, [n], [T], q, 0.05, o, lse, idx)
