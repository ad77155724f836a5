"""The paged cache: rows appended to pages and attention over them against 64-bit plain forms, and both as a session
uses them."""
import numpy as np
import pytest
import torch

import kvp_plain as plain
import paper_2606_20537_amd as cap

pytestmark = pytest.mark.gpu
NAN = float("nan")


def host(x):
    return x.detach().cpu().double().numpy()


class Step:
    """A cache of sequences of n rows, T of them new, on pages in random order; every row that no sequence holds is NaN."""

    def __init__(self, n, T, Hkv, d, page, seed=0, absent=(), columns=None, spare=3):
        self.gen = torch.Generator("cuda").manual_seed(seed)
        self.n, self.T, self.Hkv, self.d, self.page = list(n), list(T), Hkv, d, page
        need = [min(-(-m // page), columns or 1 << 24) for m in self.n]
        self.pages = sum(need) + spare
        order = torch.randperm(self.pages, generator=torch.Generator().manual_seed(seed)).int()
        self.table = torch.full((len(self.n), columns or max(need + [1]) + 1), -1, dtype=torch.int32)
        for i, m in enumerate(need):
            self.table[i, :m] = order[sum(need[:i]):sum(need[:i]) + m]
        for i, c in absent:
            self.table[i, c] = -1
        self.k, self.v = (torch.full((self.pages, page, Hkv, d), NAN, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        for i, m in enumerate(self.n):
            for r0 in range(0, min(m, need[i] * page), page):
                p = int(self.table[i, r0 // page])
                if p >= 0:
                    rows = min(page, m - r0)
                    self.k[p, :rows], self.v[p, :rows] = self.normal(rows, Hkv, d), self.normal(rows, Hkv, d)
        self.lens = torch.tensor(self.n, dtype=torch.int32, device="cuda")
        self.tok0 = torch.tensor([sum(self.T[:i]) for i in range(len(self.T) + 1)], dtype=torch.int32, device="cuda")
        self.tokens = sum(self.T)
        self.dev_table = self.table.cuda()
        self.cache = cap.kvp_cache(self.k, self.v, self.dev_table)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.gen, device="cuda").bfloat16()

    def there(self, i):
        """Which rows of sequence i lie on a page."""
        r = np.arange(min(self.n[i], self.table.shape[1] * self.page))
        t = self.table[i].numpy()[r // self.page]
        return (t >= 0) & (t < self.pages)

    def rows(self, i, x):
        """Rows [0, n) of sequence i of a pool (of absent pages: NaN), on the host."""
        r = torch.arange(min(self.n[i], self.table.shape[1] * self.page))
        if len(r) == 0:
            return np.zeros((0, self.Hkv, self.d))
        t = self.table[i, r // self.page].long()
        out = host(x[t.clamp(0, self.pages - 1).cuda(), (r % self.page).cuda()])
        out[((t < 0) | (t >= self.pages)).numpy()] = np.nan
        return out

    def check(self, q, o, lse, scale, window=0):
        G, qh, oh, lh = q.shape[1] // self.Hkv, host(q), host(o), host(lse)
        for i, (n, T) in enumerate(zip(self.n, self.T)):
            t0, there, k, v = sum(self.T[:i]), self.there(i), self.rows(i, self.k), self.rows(i, self.v)
            for t in range(T):
                rows = plain.seen_rows(n - T + t, window, there)
                for h in range(q.shape[1]):
                    want = plain.attend(qh[t0 + t, h], k[:, h // G], v[:, h // G], scale, rows)
                    assert plain.attend_near(oh[t0 + t, h], lh[t0 + t, h], want, max(1, len(rows))), (i, t, h)

    def attend(self, G, window=0, scale=None, q=None, **kw):
        scale = self.d ** -0.5 if scale is None else scale
        q = self.normal(self.tokens, self.Hkv * G, self.d) * 1.5 if q is None else q
        o, lse = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty(q.shape[:2], device="cuda")
        cap.kvp_attend(self.cache, self.lens, q, o, scale=scale, tok0=self.tok0, window=window, lse=lse, **kw)
        return q, o, lse


LENGTHS = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 200, 500, 513, 1030, 0]


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 48, 256])
def test_lengths(d, page):
    s = Step(LENGTHS, [1] * len(LENGTHS), 2, d, page, seed=d + page)
    s.check(*s.attend(2), d ** -0.5)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n", [1, 40, 255])
def test_short_caches_in_one_launch(d, n):
    s = Step([n, 0, 17], [1, 1, 1], 3, d, 16, seed=n, columns=2048 // d if d > 64 else 48)
    assert cap.kvp_attend_workspace_bytes(s.cache, 3, 6) == 0
    s.check(*s.attend(2), d ** -0.5)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_short_windows_in_one_launch(d):
    s = Step([5000, 3, 900], [1, 2, 1], 2, d, 64, seed=d)
    assert cap.kvp_attend_workspace_bytes(s.cache, 4, 4, 200) == 0 < cap.kvp_attend_workspace_bytes(s.cache, 4, 4)
    s.check(*s.attend(2, window=200), d ** -0.5, 200)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_segments_for_every_workgroup(d):
    # whole segments of up to 1024 rows; the same cut, with one row more on the table
    n = [1000, 7, 333, 0, 64] * (-(-65536 // d // 8 // 5))
    s = Step(n, [1] * len(n), 8, d, 16, seed=d, columns=64)
    assert cap.kvp_attend_workspace_bytes(s.cache, len(n), 8) == 0
    q, o, lse = s.attend(1)
    pick = [0, 1, 2, 3, 4, len(n) - 5]
    host_q, host_o, host_l = host(q[pick]), host(o[pick]), host(lse[pick])
    for j, i in enumerate(pick):
        k, v = s.rows(i, s.k), s.rows(i, s.v)
        for h in range(8):
            want = plain.attend(host_q[j, h], k[:, h], v[:, h], d ** -0.5, np.arange(n[i]))
            assert plain.attend_near(host_o[j, h], host_l[j, h], want, max(1, n[i]))
    wide = torch.cat([s.dev_table, torch.full_like(s.dev_table[:, :1], -1)], 1)
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    cap.kvp_attend(cap.kvp_cache(s.k, s.v, wide), s.lens, q, o2, scale=d ** -0.5, lse=lse2)
    assert (o2.float() - o.float()).abs().max() <= 2.0 ** -7 * o.float().abs().max()
    fine = lse.isfinite()
    assert torch.equal(fine, lse2.isfinite()) and (lse2 - lse)[fine].abs().max() <= 1e-4


@pytest.mark.parametrize("G, Hkv", [(1, 1), (1, 8), (3, 2), (8, 1), (16, 2), (17, 1), (40, 1)])
def test_heads(G, Hkv):
    s = Step([300, 90, 2000], [1, 3, 1], Hkv, 64, 32, seed=G)
    s.check(*s.attend(G), 0.125)


@pytest.mark.parametrize("d", [64, 256])
@pytest.mark.parametrize("window", [0, 1, 5, 64, 100])
def test_tokens_and_windows(d, window):
    n, T = [7, 100, 700, 33, 64, 40, 3], [7, 2, 5, 1, 0, 40, 3]
    s = Step(n, T, 2, d, 16, seed=window)
    s.check(*s.attend(3, window=window), d ** -0.5, window)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_long_sequences_are_cut_and_joined(d):
    s = Step([20000, 1, 4097, 333], [1, 1, 2, 1], 2, d, 64, seed=d)
    s.check(*s.attend(4), d ** -0.5)


def test_window_over_a_long_sequence():
    # pages before the window are gone; one token of several tiles
    n = 9000
    s = Step([n, n], [1, 6], 1, 128, 64, seed=5, absent=[(i, c) for i in (0, 1) for c in range((n - 6 - 1000) // 64)])
    s.check(*s.attend(8, window=1000), 128 ** -0.5, 1000)


def test_absent_pages_and_rows_beyond_the_table():
    s = Step([200, 90, 64, 300], [2, 1, 1, 1], 2, 64, 16, seed=2, absent=[(0, 0), (0, 7), (0, 12), (1, 5)] + [(2, c) for c in range(4)], columns=15)
    s.dev_table[3, 2] = s.pages       # no page either
    s.table[3, 2] = s.pages
    s.check(*s.attend(2), 0.125)      # (sequence 3: rows 240 .. 299 are beyond the table)


def test_tokens_before_the_first_row():
    # more tokens than rows held: the first ones see nothing
    s = Step([2, 0, 70], [5, 3, 2], 2, 128, 16, seed=9)
    q, o, lse = s.attend(2)
    s.check(q, o, lse, 128 ** -0.5)
    assert not o[:3].any() and (lse[:3] == -float("inf")).all() and not o[5:8].any()


@pytest.mark.parametrize("n_seq", [63, 64, 65, 130, 1024])
def test_many_sequences(n_seq):
    rng = np.random.default_rng(n_seq)
    n, T = rng.integers(0, 90, n_seq).tolist(), rng.integers(0, 3, n_seq).tolist()
    s = Step(n, T, 1, 64, 16, seed=n_seq, columns=40)  # (two launches)
    s.check(*s.attend(2), 0.125)


def test_one_token_for_each_sequence_without_tok0():
    s = Step([33, 700, 1, 5], [1] * 4, 2, 64, 16)
    q, o, lse = s.attend(2)
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    cap.kvp_attend(s.cache, s.lens, q, o2, scale=0.125, lse=lse2)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    o3 = torch.empty_like(o)
    cap.kvp_attend(s.cache, s.lens, q, o3, scale=0.125)  # no lse
    assert torch.equal(o, o3)
    with pytest.raises(cap.CapsuleError):
        cap.kvp_attend(s.cache, s.lens, q[:3], o[:3], scale=0.125)


@pytest.mark.parametrize("columns", [32, 100])
def test_tokens_of_no_sequence_stay(columns):
    s = Step([100, 7], [2, 1], 2, 64, 16, columns=columns)
    q, o, lse = s.normal(8, 4, 64), torch.full((8, 4, 64), 3.0, device="cuda").bfloat16(), torch.full((8, 4), 5.0, device="cuda")
    cap.kvp_attend(s.cache, s.lens, q, o, scale=0.125, tok0=s.tok0, lse=lse)
    assert (o[3:] == 3).all() and (lse[3:] == 5).all()
    s.check(q[:3], o[:3], lse[:3], 0.125)
    if columns == 100:  # the first tokens belong to none either
        o.fill_(3.0)
        cap.kvp_attend(s.cache, s.lens, q, o, scale=0.125, tok0=s.tok0 + 4, lse=lse)
        assert (o[:4] == 3).all() and (o[7:] == 3).all() and (lse[7:] == 5).all()
        s.check(q[4:7], o[4:7], lse[4:7], 0.125)


@pytest.mark.parametrize("T", [1, 3])
def test_values_that_some_tokens_do_not_see(T):
    # infinities and NaN in rows that later tokens alone see, and in a row that all see
    s = Step([80, 80], [T, T], 2, 128, 16, seed=3)
    page, row = int(s.table[0, 79 // 16]), 79 % 16
    s.v[page, row, 0, 5], s.v[page, row, 1, 77] = float("inf"), NAN
    s.v[int(s.table[1, 0]), 3, 1, 9] = NAN
    s.k[int(s.table[1, 1]), 3, 0, 9] = NAN
    q, o, lse = s.attend(2)
    for t in range(T - 1):
        assert o[t].isfinite().all()
    last = o[T - 1]
    assert last[:2, 5].isinf().all() and last[2:, 77].isnan().all() and last.isfinite().sum() == 4 * 128 - 4
    assert lse[:T].isfinite().all()
    assert o[T:, :2].isnan().all() and lse[T:, :2].isnan().all()
    assert o[T:, 2:, 9].isnan().all() and o[T:, 2:].isfinite().sum() == T * 2 * 127
    clean = Step([80, 80], [T, T], 2, 128, 16, seed=3)
    _, o2, lse2 = clean.attend(2, q=q)
    same = o.isfinite()
    assert torch.equal(o[same], o2[same]) and torch.equal(lse[:T], lse2[:T])


def wide(s, G, window=0):
    """That the call's segments have 128 query rows: its parts need more than those of fewer."""
    return cap.kvp_attend_workspace_bytes(s.cache, s.tokens, s.Hkv * G, window) > 1 << 25


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 3, 50, 300])
def test_runs_of_tokens(d, window):
    n, T = [700, 130, 1000, 64, 0, 90, 129, 43], [300, 130, 1, 64, 0, 9, 129, 43]
    s = Step(n, T, 2, d, 48, seed=window, columns=25000 if window else 1600)
    assert window or wide(s, 3)
    s.check(*s.attend(3, window=window), d ** -0.5, window)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("G, window", [(3, 0), (17, 0), (40, 700)])
def test_runs_behind_long_sequences(d, G, window):
    # more units than even parts have, and fewer; the second sequence has one tile
    s = Step([20011, 300, 4097], [320 // G, 1, 140 // G], 1, d, 64, seed=G, columns=2500)
    if not window:
        assert wide(s, G)
    s.check(*s.attend(G, window=window), d ** -0.5, window)


def test_runs_of_many_sequences():
    rng = np.random.default_rng(5)
    n = rng.integers(0, 200, 130).tolist()
    T = [int(rng.integers(0, m + 1)) if i % 3 else 0 for i, m in enumerate(n)]
    s = Step(n, T, 1, 128, 16, seed=5, columns=200)
    assert wide(s, 5)
    s.check(*s.attend(5), 128 ** -0.5)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_runs_in_one_launch(d):
    n = [100, 7, 128, 0, 64, 99] * (-(-65536 // d // 8 // 6))
    T = [40 if m else 0 for m in n]
    T[1] = 7
    s = Step(n, T, 8, d, 16, seed=d, columns=8)
    assert cap.kvp_attend_workspace_bytes(s.cache, s.tokens, 32) == 0
    q, o, lse = s.attend(4)
    few = Step.__new__(Step)  # the first six
    few.__dict__.update(s.__dict__, n=n[:6], T=T[:6])
    few.check(q, o, lse, d ** -0.5)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 1, 50, 333])
def test_runs_of_windows(d, window):
    # some with more tokens than rows, some with rows beyond the table, one to seven tiles each
    rng = np.random.default_rng(window)
    n = [1300, 20, 1120, 1160, 64, 500] + rng.integers(0, 400, 18).tolist()
    T = [110, 70, 33, 222, 64, 32] + rng.integers(60, 130, 18).tolist()
    s = Step(n, T, 2, d, 16, seed=d + window, columns=70)
    assert wide(s, 4, window)
    few = Step.__new__(Step)  # the first eight
    few.__dict__.update(s.__dict__, n=n[:8], T=T[:8])
    few.check(*s.attend(4, window=window), d ** -0.5, window)


@pytest.mark.parametrize("window", [7, 90])
def test_runs_of_windows_in_one_launch(window):
    n = [1300, 20, 900, 40, 64, 500] * 4
    T = [41, 30, 64, 40, 1, 33] * 4
    s = Step(n, T, 16, 256, 16, seed=window)
    assert cap.kvp_attend_workspace_bytes(s.cache, s.tokens, 64, window) == 0
    few = Step.__new__(Step)
    few.__dict__.update(s.__dict__, n=n[:6], T=T[:6])
    few.check(*s.attend(4, window=window), 0.0625, window)


def test_runs_on_absent_pages_and_before_the_first_row():
    # the first 150 tokens of sequence 0 see nothing, those of sequence 3 neither
    s = Step([50, 400, 500, 90], [200, 150, 40, 30], 2, 64, 16, seed=2, columns=2600, absent=[(0, 1), (1, 0), (1, 7), (1, 12), (1, 24)] + [(3, c) for c in range(6)])
    assert wide(s, 2)
    q, o, lse = s.attend(2)
    s.check(q, o, lse, 0.125)
    assert not o[:150].any() and (lse[:150] == -float("inf")).all() and not o[390:].any()
    # rows beyond the table, and packed tokens of no sequence
    short = Step([700, 640], [90, 80], 2, 256, 16, seed=3, columns=40)
    q, o, lse = short.normal(180, 8, 256), torch.full((180, 8, 256), 3.0, device="cuda").bfloat16(), torch.full((180, 8), 5.0, device="cuda")
    cap.kvp_attend(short.cache, short.lens, q, o, scale=0.0625, tok0=short.tok0 + 6, lse=lse)
    assert (o[:6] == 3).all() and (o[176:] == 3).all() and (lse[:6] == 5).all() and (lse[176:] == 5).all()
    short.check(q[6:176], o[6:176], lse[6:176], 0.0625)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_values_that_some_tokens_of_a_run_do_not_see(d):
    n, T, G = [270, 150], [200, 120], 2
    make = lambda: Step(n, T, 2, d, 16, seed=d, columns=5000)
    s, clean = make(), make()
    put = [(0, 269, 0, 5, "v", float("inf")), (0, 200, 1, 33, "v", NAN), (0, 131, 0, 6, "v", -float("inf")), (1, 149, 1, 7, "k", NAN), (1, 64, 0, 8, "v", float("inf"))]
    q, o2, lse2 = clean.attend(G)
    want, want_lse = o2.clone(), lse2.clone()
    t0 = [0, T[0]]
    for i, row, h, c, what, value in put:
        getattr(s, what)[int(s.table[i, row // 16]), row % 16, h, c] = value
        first = t0[i] + row - (n[i] - T[i])  # the packed token at that row
        mine = slice(h * G, h * G + G)
        last = t0[i] + T[i]
        if what == "v":
            want[first:last, mine, c] = value
        else:
            want[first:last, mine], want_lse[first:last, mine] = NAN, NAN
    _, o, lse = s.attend(G, q=q)
    assert wide(s, G)
    assert torch.equal(o.nan_to_num(9.0, 1e30, -1e30), want.nan_to_num(9.0, 1e30, -1e30))
    assert torch.equal(o.isnan(), want.isnan()) and torch.equal(lse.nan_to_num(9.0), want_lse.nan_to_num(9.0))


def test_a_run_out_of_strided_queries_is_reproducible():
    s = Step([900, 333], [400, 200], 2, 128, 64, seed=11, columns=1500)
    q = s.normal(600, 2, 8, 128)[:, 1]
    assert wide(s, 4)
    _, o, lse = s.attend(4, q=q)
    s.check(q, o, lse, 128 ** -0.5)
    for _ in range(3):
        _, o2, lse2 = s.attend(4, q=q)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_large_and_small_values():
    for size in (3e38, 1e-30):
        s = Step([3000, 40], [1, 1], 1, 64, 16, seed=4)
        s.v.copy_((s.v.float().clamp(-1, 1) * size).bfloat16())
        q, o, lse = s.attend(2, scale=1e-3)
        assert o.isfinite().all()
        s.check(q, o, lse, 1e-3)


def test_large_scores():
    s = Step([600, 3], [1, 2], 2, 64, 16, seed=6)
    for scale in (30.0, -30.0, 0.0):
        s.check(*s.attend(2, scale=scale), scale)
    s = Step([300, 90], [150, 60], 2, 128, 16, seed=7, columns=6000)
    assert wide(s, 2)
    for scale in (5.0, -5.0, 0.0, 1e-44):
        s.check(*s.attend(2, scale=scale), scale)


@pytest.mark.parametrize("T", [1, 100])
def test_scores_beyond_fp32(T):
    # row 3's product with the first channel of a query is 2^100, times the scale 2^30 above the range; with -2^30 below it
    s = Step([150, 40], [T, 1], 1, 64, 16, seed=7, columns=19300)
    s.k[int(s.table[0, 0]), 3, 0] = 0
    s.k[int(s.table[0, 0]), 3, 0, 0] = 2.0 ** 100
    q = s.normal(s.tokens, 3, 64) * 1e-9
    q[:, :, 0] = 1.0
    assert T == 1 or wide(s, 3)
    _, o, lse = s.attend(3, q=q, scale=2.0 ** 30)
    assert o[:T].isnan().all() and lse[:T].isnan().all() and o[T:].isfinite().all() and lse[T:].isfinite().all()
    _, o, lse = s.attend(3, q=q, scale=-2.0 ** 30)
    assert o.isfinite().all() and lse.isfinite().all()


def test_strided_queries_and_pools():
    Hkv, G, d, page = 2, 3, 128, 16
    s = Step([90, 600], [2, 1], Hkv, d, page, seed=8)
    q, o, lse = s.attend(G)
    wide = s.normal(3, 2 * Hkv * G + 5, d)
    wide[:, 1:1 + 2 * Hkv * G:2] = q
    o2 = torch.empty_like(o)
    cap.kvp_attend(s.cache, s.lens, wide[:, 1:1 + 2 * Hkv * G:2], o2, scale=d ** -0.5, tok0=s.tok0)
    assert torch.equal(o, o2)
    both = torch.stack([s.k, s.v], 1)  # [pages, 2, page, Hkv, d]
    table = torch.full((2, 60), -1, dtype=torch.int32, device="cuda")
    table[:, :s.dev_table.shape[1]] = s.dev_table
    cache = cap.kvp_cache(both[:, 0], both[:, 1], table[:, :s.dev_table.shape[1]])
    cap.kvp_attend(cache, s.lens, q, o2, scale=d ** -0.5, tok0=s.tok0)
    assert torch.equal(o, o2)


def test_pools_past_32_bits():
    # pages whose bytes lie beyond 2^32 (and elements beyond 2^32 too)
    page, Hkv, d = 1024, 8, 256
    pages = (1 << 32) // (page * Hkv * d) + 40
    k, v = (torch.empty((pages, page, Hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.tensor([[pages - 1, 0, pages // 2 + 1, pages - 3]], dtype=torch.int32, device="cuda")
    gen = torch.Generator("cuda").manual_seed(1)
    n = 3500
    at = table[0].long()
    k[at], v[at] = (torch.randn((4, page, Hkv, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    cache = cap.kvp_cache(k, v, table)
    new = torch.randn((2, 1, Hkv, d), generator=gen, device="cuda").bfloat16()
    cap.kvp_append(cache, lens, new[0], new[1])
    r = n - 1
    assert torch.equal(k[at[r // page], r % page], new[0, 0]) and torch.equal(v[at[r // page], r % page], new[1, 0])
    q = torch.randn((1, Hkv, d), generator=gen, device="cuda").bfloat16()
    o, lse = torch.empty_like(q), torch.empty((1, Hkv), device="cuda")
    cap.kvp_attend(cache, lens, q, o, scale=d ** -0.5, lse=lse)
    kh, vh = host(k[at].flatten(0, 1)[:n]), host(v[at].flatten(0, 1)[:n])
    for h in range(Hkv):
        assert plain.attend_near(host(o)[0, h], host(lse)[0, h], plain.attend(host(q)[0, h], kh[:, h], vh[:, h], d ** -0.5, np.arange(n)), n)


# ------------------------------------------------------------------ append --
@pytest.mark.parametrize("d, page", [(64, 16), (128, 48), (256, 64)])
@pytest.mark.parametrize("rot, pairs", [(None, False), (0, False), (32, False), (64, True)])
def test_append(d, page, rot, pairs):
    n, T = [1, 100, 0, 47, 600, 5], [1, 37, 0, 47, 530, 7]  # (the last: more tokens than rows)
    s = Step(n, T, 2, d, page, seed=d, absent=[(4, 3)])
    s.dev_table[1, 1] = s.table[1, 1] = s.pages + 5
    heads, extra = 5, 4  # tokens of no sequence at the end
    before = s.k.clone(), s.v.clone()
    x = s.normal(s.tokens + extra, heads + 4, d)
    q, k, v = x[:, :heads], x[:, heads:heads + 2], x[:, heads + 2:]
    kw, keys, want_q = {}, host(k), None
    if rot is not None:
        f = cap.qk_freqs(1e6, rot).cuda() if rot else None
        w = (1 + 0.2 * torch.randn(d, generator=s.gen, device="cuda")).bfloat16()
        rule = cap.qk_rule(f, wq=w, wk=w, eps=1e-6, pairs=pairs)
        q_out = torch.full((s.tokens + extra, heads, d), 7.0, device="cuda").bfloat16()
        kw = dict(rule=rule, q=q, q_out=q_out)
        pos = np.concatenate([np.arange(m - t, m) for m, t in zip(n, T)] + [np.zeros(extra)])[:, None]
        fh = None if f is None else host(f)
        keys, k_size = plain.turned(keys, host(w), pos, fh, 1e-6, 0.0, rot, pairs)
        want_q, q_size = plain.turned(host(q), host(w), pos, fh, 1e-6, 0.0, rot, pairs)
    cap.kvp_append(s.cache, s.lens, k, v, tok0=s.tok0, **kw)
    kh, vh = host(s.k), host(s.v)
    mine = np.zeros((s.pages, page), bool)
    for i in range(len(n)):
        there = s.there(i)
        for t in range(T[i]):
            r, at = n[i] - T[i] + t, sum(T[:i]) + t
            if rot is not None:
                if r >= 0:
                    assert plain.turned_near(host(q_out[at]), want_q[at], q_size[at], 2.0 ** -8)
                else:
                    assert (q_out[at] == 7).all()
            if r < 0 or not there[r]:
                continue
            p = int(s.table[i, r // page])
            mine[p, r % page] = True
            assert np.array_equal(vh[p, r % page], host(v[at]))
            if rot is None:
                assert np.array_equal(kh[p, r % page], keys[at])
            else:
                assert plain.turned_near(kh[p, r % page], keys[at], k_size[at], 2.0 ** -8)
    for now, old in ((s.k, before[0]), (s.v, before[1])):  # every other row as it was
        a, b = now[torch.from_numpy(~mine).cuda()], old[torch.from_numpy(~mine).cuda()]
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    if rot is not None:
        assert (q_out[s.tokens:] == 7).all()


def test_append_with_positions_of_its_own():
    # an image in the prompt: three axes, positions apart from the rows'
    s = Step([30, 64], [12, 20], 2, 64, 16)
    f = cap.qk_freqs(1e4, 64, [12, 10, 10], True).cuda()
    pos = torch.randint(0, 500, (32, 3), device="cuda", dtype=torch.int32, generator=s.gen)
    k, v = s.normal(32, 2, 64), s.normal(32, 2, 64)
    rule = cap.qk_rule(f)
    cap.kvp_append(s.cache, s.lens, k, v, tok0=s.tok0, rule=rule, pos=pos)
    want = torch.empty_like(k)
    cap.qk_norm_rope(rule, None, k, None, want, pos=pos)
    got = torch.cat([s.k[s.dev_table[i].long().clamp(0)].flatten(0, 1)[n - T:n] for i, (n, T) in enumerate(zip(s.n, s.T))])
    assert torch.equal(got, want)


@pytest.mark.parametrize("n_seq", [64, 65, 300, 1024])
def test_append_to_many_sequences(n_seq):
    rng = np.random.default_rng(n_seq)
    T = rng.integers(0, 4, n_seq).tolist()
    s = Step([t + int(m) for t, m in zip(T, rng.integers(0, 40, n_seq))], T, 1, 64, 16, seed=1)
    k, v = s.normal(s.tokens, 1, 64), s.normal(s.tokens, 1, 64)
    cap.kvp_append(s.cache, s.lens, k, v, tok0=s.tok0)
    row = torch.cat([s.table[i, torch.arange(n - t, n) // 16].long() * 16 + torch.arange(n - t, n) % 16 for i, (n, t) in enumerate(zip(s.n, s.T))]).cuda()
    assert torch.equal(s.k.flatten(0, 1)[row], k) and torch.equal(s.v.flatten(0, 1)[row], v)


# ------------------------------------------------------------- as it is used --
class Session:
    """One full-attention layer of a live set: its K and V buffers are the pools, each 64 rows a page."""

    def __init__(self, seed, sessions=3, rows=512, Hkv=2, G=4, d=64, rot=32):
        self.gen = torch.Generator("cuda").manual_seed(seed)
        self.Hkv, self.G, self.d, self.rows, self.sessions = Hkv, G, d, rows, sessions
        self.k, self.v = (torch.zeros((sessions, rows, Hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        table = torch.arange(sessions * rows // 64, dtype=torch.int32, device="cuda").view(sessions, -1).clone()
        pools = [x.view(-1, 64, Hkv, d) for x in (self.k, self.v)]
        self.cache = cap.kvp_cache(pools[0], pools[1], table)
        w = (1 + 0.2 * torch.randn(d, generator=self.gen, device="cuda")).bfloat16()
        self.rule = cap.qk_rule(cap.qk_freqs(1e6, rot).cuda(), wq=w, wk=w, eps=1e-6)
        self.lens = torch.zeros(sessions, dtype=torch.int32, device="cuda")
        self.tables = torch.randn((rows, (G + 2) * Hkv, d), generator=self.gen, device="cuda").bfloat16()  # what the projections give at each row

    def layer(self, x, q, o, tok0=None, workspace=None):
        """The layer on projections x [tokens, heads + 2 kv heads, d] of the tokens that lens and tok0 tell."""
        h = self.G * self.Hkv
        cap.kvp_append(self.cache, self.lens, x[:, h:h + self.Hkv], x[:, h + self.Hkv:], tok0=tok0, rule=self.rule, q=x[:, :h], q_out=q)
        cap.kvp_attend(self.cache, self.lens, q, o, scale=self.d ** -0.5, tok0=tok0, workspace=workspace)

    def prefill(self, a, b):
        """Rows [a, b) of every session."""
        T = b - a
        x = self.tables[a:b].repeat(self.sessions, 1, 1)
        x = (x.float() * torch.arange(1, self.sessions + 1, device="cuda").repeat_interleave(T)[:, None, None]).bfloat16()
        self.lens.fill_(b)
        tok0 = torch.arange(self.sessions + 1, dtype=torch.int32, device="cuda") * T
        q = torch.empty((len(x), self.G * self.Hkv, self.d), dtype=torch.bfloat16, device="cuda")
        o = torch.empty_like(q)
        self.layer(x, q, o, tok0)
        return o.view(self.sessions, T, -1)


def test_session_restored_and_continued():
    s = Session(1)
    cold = s.prefill(0, 150)
    sets = [cap.cap_set_create([("k", s.k[i], s.Hkv * s.d * 2, s.rows, cap.CAP_KIND_POSITIONAL),
                                ("v", s.v[i], s.Hkv * s.d * 2, s.rows, cap.CAP_KIND_POSITIONAL)], 64, 7) for i in range(s.sessions)]
    arena, caps = [], []
    for c in sets:
        cap.cap_set_set_position(c, 128)
        arena.append(torch.empty(cap.capsule_bytes(c, 128), dtype=torch.uint8, device="cuda"))
        caps.append(cap.capsule_snapshot(c, 128, 3, arena[-1]))
    after = [s.prefill(r, r + 1) for r in range(150, 180)]
    rows = s.k.clone(), s.v.clone()
    s.k.fill_(NAN)
    s.v.fill_(NAN)
    for c, live in zip(caps, sets):
        assert cap.capsule_restore(c, live, 3) == 128
    rest = s.prefill(128, 150)
    again = [s.prefill(r, r + 1) for r in range(150, 180)]
    torch.cuda.synchronize()
    assert torch.equal(s.k[:, :180], rows[0][:, :180]) and torch.equal(s.v[:, :180], rows[1][:, :180])
    assert all(torch.equal(a, b) for a, b in zip(after, again))
    # the remainder's rows see the same keys; their sums are divided otherwise
    assert (rest - cold[:, 128:]).float().abs().max() <= 2.0 ** -6 * cold.float().abs().max()
    # a fork at a page's boundary: the child's table names the parent's pages
    table = s.cache.tensors[2]
    table[2, :2] = table[0, :2]
    s.lens.copy_(torch.tensor([0, 0, 128], dtype=torch.int32))
    q = torch.randn((3, s.G * s.Hkv, s.d), generator=s.gen, device="cuda").bfloat16()
    o, o2 = torch.empty_like(q), torch.empty_like(q)
    cap.kvp_attend(s.cache, s.lens, q, o, scale=0.125)
    s.k[2, :128], s.v[2, :128] = s.k[0, :128], s.v[0, :128]
    table[2, :2] = torch.tensor([2 * s.rows // 64, 2 * s.rows // 64 + 1], dtype=torch.int32)
    cap.kvp_attend(s.cache, s.lens, q, o2, scale=0.125)
    assert torch.equal(o, o2) and not o[:2].any()


def test_decode_graph_goes_on_with_the_sequences():
    eager, graphed = Session(2), Session(2)
    for s in (eager, graphed):
        s.prefill(0, 60)
    x = torch.zeros((3, (eager.G + 2) * eager.Hkv, eager.d), dtype=torch.bfloat16, device="cuda")
    q, o = (torch.empty((3, eager.G * eager.Hkv, eager.d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    work = [torch.empty(max(16, cap.kvp_attend_workspace_bytes(graphed.cache, 3, 8)), dtype=torch.uint8, device="cuda") for _ in range(2)]
    graphs = []
    for w in work:  # two graphs, each with a workspace of its own
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            graphed.layer(x, q, o, workspace=w)
        graphs.append(g)
    eo = torch.empty_like(o)
    eq = torch.empty_like(q)
    for step in range(60, 80):
        x.copy_(torch.randn(x.shape, generator=eager.gen, device="cuda"))
        for s in (eager, graphed):
            s.lens.fill_(step + 1)
        graphed.lens[1] = eager.lens[1] = 0 if step % 3 == 0 else step + 1  # a session that waits
        graphs[step % 2].replay()
        eager.layer(x, eq, eo)
        torch.cuda.synchronize()
        assert torch.equal(o, eo), step
        assert torch.equal(eager.k, graphed.k) and torch.equal(eager.v, graphed.v)


def test_graph_of_a_run_goes_on_with_the_sequences():
    s = Step([1500, 900, 700], [200, 60, 40], 2, 128, 16, seed=12, columns=1600)
    assert wide(s, 4)
    q, o, lse = s.normal(300, 8, 128), torch.zeros((300, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((300, 8), device="cuda")
    work = torch.empty(cap.kvp_attend_workspace_bytes(s.cache, 300, 8, 0), dtype=torch.uint8, device="cuda")
    call = lambda o, lse, **kw: cap.kvp_attend(s.cache, s.lens, q, o, scale=0.1, tok0=s.tok0, lse=lse, **kw)
    call(o, lse, workspace=work)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(o, lse, workspace=work)
    for n, t in (([1500, 900, 700], [200, 60, 40]), ([1, 0, 600], [1, 0, 299]), ([0, 0, 0], [0, 0, 0]), ([300, 10, 0], [300, 0, 0]), ([1499, 5, 250], [10, 5, 250])):
        s.lens.copy_(torch.tensor(n, dtype=torch.int32))
        s.tok0.copy_(torch.tensor([sum(t[:i]) for i in range(4)], dtype=torch.int32))
        work.fill_(0xFF)
        eo, el = torch.full_like(o, 2.0), torch.full_like(lse, 2.0)
        o.fill_(2.0)
        lse.fill_(2.0)
        g.replay()
        call(eo, el)
        torch.cuda.synchronize()
        assert torch.equal(o, eo) and torch.equal(lse, el), n
        s.n, s.T = n, t
        s.check(q[:sum(t)], o[:sum(t)], lse[:sum(t)], 0.1)
        assert (o[sum(t):] == 2).all() and (lse[sum(t):] == 2).all()


def test_on_another_stream_with_its_own_workspace():
    s = Step([3000, 5], [1, 1], 2, 128, 16, seed=1)
    q, o, lse = s.attend(4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    for _ in range(3):
        cap.kvp_attend(s.cache, s.lens, q, o2, scale=128 ** -0.5, tok0=s.tok0, lse=lse2, stream=side)
        q2, o3, _ = s.attend(4, q=q)
    torch.cuda.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2) and torch.equal(o, o3)


def test_refusals_on_the_gpu():
    s = Step([30], [1], 1, 64, 16)
    q = s.normal(1, 2, 64)
    with pytest.raises(ValueError, match="of shape"):
        cap.kvp_attend(s.cache, s.lens, q[..., :32], q, scale=1.0)
    with pytest.raises(ValueError, match="lens"):
        cap.kvp_attend(s.cache, s.lens.long(), q, torch.empty_like(q), scale=1.0)
    with pytest.raises(ValueError, match="tok0"):
        cap.kvp_attend(s.cache, s.lens, q, torch.empty_like(q), scale=1.0, tok0=s.lens)
    with pytest.raises(cap.CapsuleError):
        cap.kvp_attend(s.cache, s.lens, q, q, scale=1.0)  # in place
    with pytest.raises(cap.CapsuleError):
        cap.kvp_attend(s.cache, None, q, torch.empty_like(q), scale=1.0)
    with pytest.raises(ValueError, match="go with a rule"):
        cap.kvp_append(s.cache, s.lens, s.normal(1, 1, 64), s.normal(1, 1, 64), q=q)
    with pytest.raises(cap.CapsuleError):
        cap.kvp_append(s.cache, s.lens, s.k[0, :1], s.normal(1, 1, 64))
