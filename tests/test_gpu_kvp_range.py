"""Attention over pages at the ends of the numbers' range, in tiles of each size, in one launch and in two."""
import numpy as np
import pytest
import torch

import kvp_plain as plain
import paper_2606_20537_amd as cap
from kvp_plan import plan_of
from test_gpu_kvp import Step, host

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")

# sequences' rows, tokens, query heads of a KV head and columns of 16 rows for tiles of 16, 32 and 128 rows, dealt out in parts, and whole ones
CALLS = {"16": ([3000, 1, 40], [1, 1, 1], 2, 260), "32": ([3000, 40], [5, 5], 4, 4096), "128": ([900, 90], [150, 60], 2, 6000),
         "whole": ([250, 1, 40], [1, 1, 2], 2, 16), "whole 128": ([128, 60], [100, 40], 4, 8)}


def step(call, d, seed):
    n, T, G, columns = CALLS[call]
    many = call == "whole 128"  # enough segments for every workgroup
    s = Step(n * (32 if many else 1), T * (32 if many else 1), 16 if many else 2, d, 16, seed=seed, columns=columns)
    tile, mode = plan_of(s, G)[:2]
    assert (mode == "whole") == call.startswith("whole") and (call == "whole" or tile == int(call.split()[-1]))
    if many:
        s.n, s.T = s.n[:2], s.T[:2]  # (those that are checked)
    return s, G


def near(o, want, mass, size, lse, n):
    """As attend_near of the plain form, but small values have only what fp32's smallest step costs: each of the n products
    with hi and lo, the n / 32 + 96 sums and the quotient is off by 2^-150 at most besides, and the sum of the weights is 1 at least; the output is off
    by half a step of bf16, 2^-134 at least.  Scores are taken from a reference that is 8 below their maximum at most."""
    dx = 2.0 ** -16 * size + 2.0 ** -22 * (abs(lse) + size + 8)
    steps = (n / 32 + 96) * 2.0 ** -24
    far = mass * (2.0 ** -16 + 2 * dx + 2 * steps) + (3 * n + 97) * 2.0 ** -150
    far = far + np.maximum(2.0 ** -8 * (np.abs(want) + far), 2.0 ** -134)
    return (np.abs(o - want) <= far).all()


def check(s, q, o, G, scale, channels=slice(None)):
    qh, oh = host(q), host(o)
    for i, (n, T) in enumerate(zip(s.n, s.T)):
        t0, k, v = sum(s.T[:i]), s.rows(i, s.k), s.rows(i, s.v)
        for t in sorted({0, T // 2, T - 1}):
            for h in range(0, q.shape[1], 3):
                rows = np.arange(n - T + t + 1)
                want, lse, mass, size = plain.attend(qh[t0 + t, h], k[:, h // G], v[:, h // G], scale, rows)
                assert near(oh[t0 + t, h][channels], want[channels], mass[channels], size, lse, len(rows)), (i, t, h)


@pytest.mark.parametrize("call", list(CALLS))
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("size", [2.0 ** -96, 2.0 ** -112, 1e-36, 2.0 ** -126])
def test_small_values(call, d, size):
    s, G = step(call, d, 4)
    s.v.copy_((s.v.float().clamp(-2, 2) * size).bfloat16())
    q, o, _ = s.attend(G, scale=0.02)
    check(s, q, o, G, 0.02)


def test_one_row_is_its_value():
    # the mean of one row is that row, of whatever size
    s = Step([1] * 40, [1] * 40, 1, 64, 16, seed=1, columns=260)
    size = 2.0 ** torch.arange(-125, 123, 6.35, device="cuda")[:40]
    for i in range(40):
        s.v[int(s.table[i, 0]), 0] = (s.v[int(s.table[i, 0]), 0].float().clamp(-1.9, 1.9) * size[i]).bfloat16()
    q, o, _ = s.attend(2)
    want = torch.stack([s.v[int(s.table[i, 0]), 0].expand(2, 64) for i in range(40)])
    assert torch.equal(o, want)


@pytest.mark.parametrize("call", list(CALLS))
@pytest.mark.parametrize("d", [64, 128, 256])
def test_small_values_beside_large_ones(call, d):
    # sums of every other channel pass fp32's range, their means do not
    s, G = step(call, d, 5)
    size = torch.tensor([3e38, 1e-36], device="cuda").repeat(d // 2)
    s.v.copy_(((1 - 0.3 * s.v.float().clamp(-1, 1).abs()) * size).bfloat16())
    q, o, lse = s.attend(G, scale=0.02)
    assert o[:sum(s.T)].isfinite().all() and lse[:sum(s.T)].isfinite().all()
    check(s, q, o, G, 0.02)


@pytest.mark.parametrize("call", list(CALLS))
@pytest.mark.parametrize("d", [64, 128, 256])
def test_large_values_of_both_signs(call, d):
    # sums that pass the range upwards and downwards (NaN, not an infinity), and scores that grow by the row, so that weights stand above 1 for a while
    s, G = step(call, d, 7)
    s.v.copy_(((1 - 0.3 * s.v.float().clamp(-1, 1).abs()) * 3.3e38 * s.v.float().sign()).bfloat16())
    for i, n in enumerate(s.n):
        r = torch.arange(min(n, s.table.shape[1] * s.page))
        at = s.table[i, r // s.page].long().cuda(), (r % s.page).cuda()
        s.k[at[0], at[1], :, 0] = (0.01 * r.cuda()).bfloat16()[:, None]
    q = s.normal(s.tokens, s.Hkv * G, d)
    q[:, :, 0] = 1.0
    q, o, lse = s.attend(G, scale=0.5, q=q)
    assert o[:sum(s.T)].isfinite().all() and lse[:sum(s.T)].isfinite().all()
    check(s, q, o, G, 0.5)


@pytest.mark.parametrize("call", list(CALLS))
@pytest.mark.parametrize("d", [64, 128, 256])
def test_infinities_beside_small_values(call, d):
    s, G = step(call, d, 6)
    s.v.copy_((s.v.float().clamp(-2, 2) * 1e-36).bfloat16())
    page = int(s.table[0, 0])
    s.v[page, 0, 0, 5], s.v[page, 0, 0, 17], s.v[page, 0, 0, 40] = INF, -INF, NAN
    q, o, lse = s.attend(G, scale=0.02)
    mine = o[:s.T[0], :G]
    assert (mine[..., 5] == INF).all() and (mine[..., 17] == -INF).all() and mine[..., 40].isnan().all()
    assert mine.isfinite().sum() == mine.numel() - 3 * s.T[0] * G and o[:s.T[0], G:].isfinite().all() and o[s.T[0]:sum(s.T)].isfinite().all()
    assert lse[:sum(s.T)].isfinite().all()
    s.v[page, 0, 0, [5, 17, 40]] = 0
    check(s, q, o, G, 0.02, [c for c in range(d) if c not in (5, 17, 40)])


@pytest.mark.parametrize("G, columns, tile", [(2, 4, 16), (2, 300, 16), (20, 4096, 32)])
def test_weights_keep_24_bits(G, columns, tile):
    # Two rows with scores 0 and -s, s of 8 bits, and values 1 and -1: o = tanh(s / 2), small beside the sum of weights.  Two's
    # weight w is off by an exponential (2^-23) and its parts (2^-23), half of which reach o; six products' sums of 1 at most
    # by 2^-23 each, halved by the quotient, and the sum of weights by 2^-24: below 12 * 2^-24.  Then the output's rounding.
    n_seq = 128
    s = Step([2] * n_seq, [1] * n_seq, 1, 64, 16, columns=columns)
    assert plan_of(s, G)[0] == tile
    at = s.table[:, 0].long().cuda()
    s.k[at, :2], s.v[at, :2] = 0, 0
    s.k[at, 1, 0, 0], s.v[at, 0, 0, :], s.v[at, 1, 0, :] = -1, 1, -1
    x = (1 + torch.arange(n_seq, device="cuda") / 128) * 2.0 ** -13
    q = torch.zeros((n_seq, G, 64), device="cuda")
    q[:, :, 0] = x[:, None] * 2.0 ** torch.arange(-1, 1, device="cuda").repeat(G // 2)
    q, o, _ = s.attend(G, scale=1.0, q=q.bfloat16())
    want = np.tanh(host(q)[..., :1] / 2)
    assert (np.abs(host(o) - want) <= 12 * 2.0 ** -24 + 2.0 ** -8 * want).all()


@pytest.mark.parametrize("n", [90, (1 << 24) - 5, 1 << 24])
def test_a_window_over_the_widest_table(n):
    # 1024 sequences of 8 KV heads and 2^24 rows: a window's units are few, however many the table has
    n_seq, Hkv, d, page, window = 1024, 8, 64, 1 << 14, 100
    gen = torch.Generator("cuda").manual_seed(3)
    k, v = (torch.randn((3, page, Hkv, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    table = torch.full((n_seq, 1024), -1, dtype=torch.int32, device="cuda")
    at = torch.arange(n_seq, device="cuda") % 3
    table[:, (n - 1) // page] = at.int()  # (the window lies on one page)
    cache = cap.kvp_cache(k, v, table)
    q = torch.randn((n_seq, Hkv, d), generator=gen, device="cuda").bfloat16()
    o, lse = torch.empty_like(q), torch.empty((n_seq, Hkv), device="cuda")
    lens = torch.full((n_seq,), n, dtype=torch.int32, device="cuda")
    cap.kvp_attend(cache, lens, q, o, scale=0.125, window=window, lse=lse)
    rows = np.arange(max(0, n - window), n) % page
    kh, vh, qh, oh, lh = host(k), host(v), host(q), host(o), host(lse)
    for i in (0, 1, 500, 1023):
        for h in range(Hkv):
            want = plain.attend(qh[i, h], kh[i % 3, :, h], vh[i % 3, :, h], 0.125, rows)
            assert plain.attend_near(oh[i, h], lh[i, h], want, len(rows)), (i, h)


@pytest.mark.parametrize("call", list(CALLS))
@pytest.mark.parametrize("scale", [2.0 ** -130, -2.0 ** -130])
def test_products_beyond_fp32(call, scale):
    # q . k of row 2 is +-2^140, which the small scale comes after: above the range the row is NaN, below it row 2 counts as none
    s, G = step(call, 64, 8)
    page = int(s.table[0, 0])
    s.k[page, 2] = 0
    s.k[page, 2, :, 0] = 2.0 ** 70
    q = s.normal(s.tokens, s.Hkv * G, 64)
    for sign in (1.0, -1.0):
        q[:, :, 0] = sign * 2.0 ** 70
        _, o, lse = s.attend(G, q=q, scale=scale)
        first = s.T[0]
        if sign * scale > 0:
            assert o[:first].isnan().all() and lse[:first].isnan().all()
        else:
            assert o[:first].isfinite().all() and lse[:first].isfinite().all()
            n, T = s.n[0], s.T[0]
            v = s.rows(0, s.v)[:, 0]
            want = np.delete(v, 2, 0)[:n - 1].mean(0)  # the last token sees all other rows alike
            assert np.abs(host(o)[T - 1, 0] - want).max() <= 2.0 ** -7 * np.abs(v).max()


def test_pools_with_dimensions_of_one():
    s = Step([90, 7], [1, 1], 1, 64, 16, seed=9)
    q, o, lse = s.attend(4)
    k = s.k.transpose(1, 2).contiguous().transpose(1, 2)  # [pages, head, rows, channels] of one head
    o2 = torch.empty_like(o)
    cap.kvp_attend(cap.kvp_cache(k, s.v, s.dev_table), s.lens, q, o2, scale=0.125, tok0=s.tok0)
    assert torch.equal(o, o2)
    both = torch.stack([s.k[:1], s.k[1:2], s.v[:1]], 1)  # one page, apart from others
    table = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    lens = torch.tensor([5], dtype=torch.int32, device="cuda")
    both[:, :, :5] = s.normal(1, 3, 5, 1, 64)
    o3, o4 = torch.empty_like(o[:1]), torch.empty_like(o[:1])
    cap.kvp_attend(cap.kvp_cache(both[:, 0], both[:, 2].clone(), table), lens, q[:1], o3, scale=0.125)
    cap.kvp_attend(cap.kvp_cache(both[:, 0].clone(), both[:, 2].clone(), table), lens, q[:1], o4, scale=0.125)
    assert torch.equal(o3, o4) and o3.isfinite().all()


def test_a_scale_that_no_field_holds():
    s = Step([30], [1], 1, 64, 16)
    for scale in (1e39, -1e39, "1"):
        with pytest.raises(ValueError, match="scale"):
            s.attend(2, scale=scale)
    with pytest.raises(cap.CapsuleError):
        s.attend(2, scale=INF)
