"""Attention over pages in tiles of each size and each way of dealing out the work, every row against the 64-bit form."""
import math

import numpy as np
import pytest
import torch

import paper_2606_20537_amd as cap
from kvp_plan import places, plan_of
from test_gpu_kvp import Step

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")

HKV = 4
GROUP = {16: 4, 32: 8, 128: 4}
# tokens of sequences in turn: last tiles of one to all rows, tiles of odd and even number, sequences that wait
TOKENS = {16: [1, 2, 4, 3, 0, 1], 32: [3, 5, 4, 3, 4, 2], 128: [40, 97, 33, 64, 0, 131, 7, 160]}


def make(tile, mode, d, seed=0):
    rng = np.random.default_rng(seed + tile + d)
    of = TOKENS[tile]
    per = sum(-(-t * GROUP[tile] // tile) for t in of) * HKV / len(of)  # segments of a sequence
    count = {"parts": len(of), "whole": places(d, 16) // HKV + 3, "runs": int(1.1 * places(d, tile) / per) + 2}[mode]
    T = [of[i % len(of)] for i in range(count)]
    n = rng.integers(1, 700, count).tolist()
    n[3], n[1] = 1, T[1]  # fewer rows than tokens, and as many
    columns = 64
    if mode == "parts":
        n[0], columns = 5003, {16: 400, 32: 3100, 128: 3000}[tile]
    elif mode == "runs":  # one long sequence, whose segments several workgroups share, and one with rows beyond the table
        columns = 1300
        n[2], n[-1] = 20011, 1300 * 16 + 90
        T[-1] = of[0]
    else:
        n[2] = 1100
    s = Step(n, T, HKV, d, 16, seed=seed, columns=columns)
    assert plan_of(s, GROUP[tile])[:2] == (tile, mode)
    return s


def plain_rows(s, i, q, scale, window):
    """Sequence i's tokens in 64 bits on the GPU: o, lse, sum of weight times |v|, largest sum of a score's products, rows seen."""
    n, T, G = s.n[i], s.T[i], q.shape[1] // s.Hkv
    t0, there = sum(s.T[:i]), torch.from_numpy(s.there(i)).cuda()
    k, v = (torch.from_numpy(s.rows(i, x)).cuda() for x in (s.k, s.v))
    k[~there], v[~there] = 0, 0
    r, pos = torch.arange(len(there), device="cuda"), torch.arange(n - T, n, device="cuda")[:, None]
    seen = (r <= pos) & there
    if window:
        seen &= r > pos - window
    seen = seen.repeat_interleave(G, 0)
    out = [[] for _ in range(4)]
    for h in range(s.Hkv):
        x = q[t0:t0 + T, h * G:(h + 1) * G].double().reshape(T * G, s.d)
        score = (scale * (x @ k[:, h].t().contiguous())).masked_fill(~seen, -INF)
        size = (abs(scale) * (x.abs() @ k[:, h].abs().t().contiguous())).masked_fill(~seen, 0.0)
        lse = torch.logsumexp(score, 1) if len(there) else torch.full((T * G,), -INF, dtype=torch.float64, device="cuda")
        p = (score - lse[:, None]).exp().masked_fill(~seen, 0.0)
        for to, y in zip(out, (p @ v[:, h], lse, p @ v[:, h].abs(), size.amax(1) if len(there) else lse * 0)):
            to.append(y.view(T, G, *y.shape[1:]))
    return [torch.cat(x, 1) for x in out] + [seen.sum(1).view(T, G)[:, :1]]


def check(s, q, o, lse, scale, window, some=None):
    """All tokens of the sequences `some` (None: all), with the bounds of kvp_plain.attend_near."""
    for i in range(len(s.n)) if some is None else some:
        T, t0 = s.T[i], sum(s.T[:i])
        if T == 0:
            continue
        want, want_lse, mass, size, rows = plain_rows(s, i, q, scale, window)
        got, got_lse = o[t0:t0 + T].double(), lse[t0:t0 + T].double()
        none = want_lse == -INF
        assert (got_lse[none] == -INF).all() and not got[none].any(), i
        base = want_lse.masked_fill(none, 0.0)
        dx = 2.0 ** -16 * size + 2.0 ** -22 * (base.abs() + size + 32)
        steps = (rows / 32 + 96) * 2.0 ** -24
        far = mass * (2.0 ** -16 + 2 * dx + 2 * steps)[..., None] + 1e-37
        assert ((got - want).abs() <= far + 2.0 ** -8 * (want.abs() + far)).all(), i
        assert ((got_lse - want_lse).abs() <= dx + steps + 2.0 ** -22 * (1 + base.abs()))[~none].all(), i


def chosen(s):
    """The first sequences, and those about the chunks of 64 and the end."""
    return sorted({i for i in list(range(9)) + [62, 63, 64, 65, 127, 128] + [len(s.n) - 2, len(s.n) - 1] if 0 <= i < len(s.n)})


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("mode", ["parts", "runs", "whole"])
@pytest.mark.parametrize("tile", [16, 32, 128])
def test_every_tile_and_mode(tile, mode, d):
    s = make(tile, mode, d)
    q, o, lse = s.attend(GROUP[tile])
    check(s, q, o, lse, d ** -0.5, 0, chosen(s))


@pytest.mark.parametrize("window", [1, 70, 3000])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("mode", ["parts", "runs", "whole"])
@pytest.mark.parametrize("tile", [16, 32, 128])
def test_every_tile_and_mode_with_a_window(tile, mode, d, window):
    # (the window may change the way that work is dealt out)
    s = make(tile, mode, d, seed=window)
    q, o, lse = s.attend(GROUP[tile], window=window)
    check(s, q, o, lse, d ** -0.5, window, chosen(s))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("mode", ["parts", "runs", "whole"])
@pytest.mark.parametrize("tile", [16, 32, 128])
def test_values_that_later_tokens_see(tile, mode, d):
    # infinities and NaN in the newest rows of every sequence: tokens before them keep every bit, later ones have them in their channels
    s = make(tile, mode, d, seed=5)
    G, t0 = GROUP[tile], np.cumsum([0] + s.T)
    q, clean, clean_lse = s.attend(G)
    want, put = clean.clone(), []
    for i in chosen(s):
        n, T = s.n[i], s.T[i]
        for back, h, c, value in ((1, 0, 5, INF), (2, 1, 9, NAN), (T // 2, 2, 17, -INF), (T, 3, 33, NAN)):
            row, first = n - back, max(0, T - back)  # the first token that sees it
            if row < 0 or back < 1 or back > T or row >= s.table.shape[1] * 16:
                continue
            s.v[int(s.table[i, row // 16]), row % 16, h, c] = value
            want[t0[i] + first:t0[i] + T, h * G:(h + 1) * G, c] = value
            put.append(value)
    assert len(put) > 8
    _, o, lse = s.attend(G, q=q)
    assert torch.equal(o.isnan(), want.isnan()) and torch.equal(o.nan_to_num(9.0, INF, -INF), want.nan_to_num(9.0, INF, -INF))
    assert torch.equal(lse, clean_lse)


@pytest.mark.parametrize("tile", [16, 32, 128])
def test_runs_are_reproducible(tile):
    s = make(tile, "runs", 128, seed=2)
    q, o, lse = s.attend(GROUP[tile])
    for _ in range(3):
        _, o2, lse2 = s.attend(GROUP[tile], q=q)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_a_long_prompt(d):
    # equal runs over pairs of one sequence's tiles: an odd number of them, behind rows and behind none
    for before in (0, 1003):
        T = 2085
        s = Step([before + T], [T], HKV, d, 64, seed=d, columns=500 if d == 256 else 300)
        tile, mode = plan_of(s, 16)[:2]
        assert tile == 128 and mode == "runs" and math.ceil(T * 16 / 128) % 2 == 1
        q, o, lse = s.attend(16)
        check(s, q, o, lse, d ** -0.5, 0)
