"""Refusals of qk_norm_rope, kvp_append and kvp_attend, on the host: the status codes of the C ABI with addresses that
are never used, what the binding refuses by itself, and the frequencies of a rule."""
import ctypes as ct

import numpy as np
import pytest
import torch

import paper_2606_20537_amd as cap
from paper_2606_20537_amd import _native as N

A = 1 << 44  # addresses far apart; nothing reads them


def at(i):
    return A + (i << 38)


def rows(i, token=0, head=0):
    return N.qk_rows(at(i) if i is not None else 0, token, head)


def rule(**kw):
    f = dict(freqs=at(20), wq=at(21), wk=at(22), rot=64, axes=1, eps=1e-6, w_add=0.0, w_dtype=cap.CAP_DTYPE_BF16, flags=cap.QK_NORM)
    return N.qk_rule_args(**{**f, **kw})


def cache(**kw):
    f = dict(k=at(10), v=at(11), table=at(12), page_stride=0, table_stride=0, pages=100, page=64, columns=16, n_seq=3, kv_heads=4, d=128,
             reserved=0)
    return N.kvp_cache_args(**{**f, **kw})


def call(name, c=None, r=None, **kw):
    r = rule() if r is None else r
    c = cache() if c is None else c
    if name == "qk_norm_rope":
        f = dict(rule=ct.addressof(r), q=rows(1), k=rows(2), q_out=rows(3), k_out=rows(4), pos=at(5), tokens=7, heads=8, kv_heads=2, d=128,
                 dtype=cap.CAP_DTYPE_BF16)
        a = N.qk_norm_rope_args(**{**f, **kw})
    elif name == "kvp_append":
        f = dict(cache=ct.addressof(c), lens=at(13), tok0=at(14), rule=ct.addressof(r), k=rows(1), v=rows(2), q=rows(3), q_out=rows(4), pos=at(5),
                 tokens=7, heads=8, reserved=0)
        a = N.kvp_append_args(**{**f, **kw})
    else:
        f = dict(cache=ct.addressof(c), lens=at(13), tok0=at(14), q=rows(1), o=at(2), lse=at(3), workspace=at(4), workspace_bytes=1 << 33, tokens=7,
                 heads=8, window=0, scale=1.0, reserved=0)
        a = N.kvp_attend_args(**{**f, **kw})
    return getattr(cap.load(), name)(ct.byref(a), None)


ALL = ["qk_norm_rope", "kvp_append", "kvp_attend"]
PAGED = ALL[1:]
INVAL, UNSUP, ALIGN, SIZE = cap.CAP_E_INVAL, cap.CAP_E_UNSUPPORTED, cap.CAP_E_ALIGN, cap.CAP_E_SIZE


def test_null_arguments():
    for name in ALL:
        assert getattr(cap.load(), name)(None, None) == INVAL
    assert call("qk_norm_rope", rule=0) == INVAL
    for name in PAGED:
        assert call(name, cache=0) == INVAL
        assert call(name, lens=0) == INVAL
        assert call(name, reserved=1) == INVAL


@pytest.mark.parametrize("name", ALL[:2])
@pytest.mark.parametrize("want, kw", [
    (INVAL, dict(flags=4)), (INVAL, dict(rot=-16)), (INVAL, dict(axes=0)), (INVAL, dict(axes=-1)), (INVAL, dict(freqs=0)), (UNSUP, dict(rot=24)),
    (UNSUP, dict(rot=144)), (UNSUP, dict(axes=9)), (INVAL, dict(w_dtype=5)), (INVAL, dict(eps=0.0)), (INVAL, dict(eps=1e-21)),
    (INVAL, dict(eps=float("inf"))), (INVAL, dict(eps=float("nan"))), (INVAL, dict(w_add=float("inf"))), (ALIGN, dict(freqs=at(20) + 4)),
    (ALIGN, dict(wq=at(21) + 8)), (ALIGN, dict(wk=at(22) + 2)),
])
def test_refused_rules(name, want, kw):
    assert call(name, r=rule(**kw)) == want


@pytest.mark.parametrize("want, kw", [
    (INVAL, dict(tokens=-1)), (INVAL, dict(heads=-1)), (INVAL, dict(kv_heads=-1)), (INVAL, dict(d=0)), (INVAL, dict(dtype=2)), (UNSUP, dict(d=120)),
    (UNSUP, dict(d=528)), (UNSUP, dict(tokens=1 << 28)), (INVAL, dict(q=rows(None))), (INVAL, dict(q_out=rows(None))), (INVAL, dict(k=rows(None))),
    (INVAL, dict(k_out=rows(None))), (INVAL, dict(pos=0)), (ALIGN, dict(pos=at(5) + 2)), (INVAL, dict(q=rows(1, 1016))), (INVAL, dict(q=rows(1, 0, 120))),
    (INVAL, dict(q=rows(1, -1024))), (ALIGN, dict(q=rows(1, 1028))), (ALIGN, dict(k_out=rows(4, 0, 132))), (UNSUP, dict(q=rows(1, (1 << 30) + 8))),
    (UNSUP, dict(k=rows(2, 0, (1 << 30) + 8))), (ALIGN, dict(q=N.qk_rows(at(1) + 8, 0, 0))), (SIZE, dict(q=N.qk_rows((1 << 64) - 1024, 0, 0))),
])
def test_refused_rotations(want, kw):
    assert call("qk_norm_rope", **kw) == want


def test_rotations_with_nothing_to_do():
    assert call("qk_norm_rope", tokens=0) == cap.CAP_OK
    assert call("qk_norm_rope", heads=0, kv_heads=0) == cap.CAP_OK
    assert call("kvp_append", tokens=0) == cap.CAP_OK
    assert call("kvp_attend", tokens=0) == cap.CAP_OK
    empty = cache(n_seq=0, table=0)
    for name in PAGED:
        assert call(name, c=empty) == cap.CAP_OK


@pytest.mark.parametrize("name", PAGED)
@pytest.mark.parametrize("want, kw", [
    (INVAL, dict(pages=-1)), (INVAL, dict(page=0)), (INVAL, dict(columns=0)), (INVAL, dict(n_seq=-1)), (INVAL, dict(kv_heads=0)), (INVAL, dict(d=0)),
    (UNSUP, dict(d=96)), (UNSUP, dict(page=24)), (UNSUP, dict(n_seq=cap.KVP_MAX_SEQ + 1)), (UNSUP, dict(pages=1 << 31)), (UNSUP, dict(columns=1 << 19)),
    (UNSUP, dict(kv_heads=1 << 20)), (INVAL, dict(page_stride=64 * 512 - 8)), (ALIGN, dict(page_stride=64 * 512 + 4)), (UNSUP, dict(page_stride=1 << 41)),
    (INVAL, dict(table_stride=15)), (INVAL, dict(table=0)), (INVAL, dict(k=0)), (INVAL, dict(v=0)), (ALIGN, dict(k=at(10) + 8)), (ALIGN, dict(table=at(12) + 2)),
    (INVAL, dict(reserved=1)), (SIZE, dict(k=(1 << 64) - 4096)), (SIZE, dict(pages=(1 << 31) - 1, page_stride=1 << 40)),
])
def test_refused_caches(name, want, kw):
    assert call(name, c=cache(**kw)) == want


@pytest.mark.parametrize("name", PAGED)
@pytest.mark.parametrize("want, kw", [
    (INVAL, dict(tokens=-1)), (INVAL, dict(tok0=0)), (ALIGN, dict(lens=at(13) + 2)), (ALIGN, dict(tok0=at(14) + 1)), (UNSUP, dict(tokens=1 << 27)),
    (SIZE, dict(lens=(1 << 64) - 4)),
])
def test_refused_steps(name, want, kw):
    assert call(name, **kw) == want


def test_refused_appends():
    for x in ("k", "v", "q", "q_out"):
        assert call("kvp_append", **{x: rows(None)}) == INVAL
        assert call("kvp_append", **{x: N.qk_rows(at(30) + 8, 0, 0)}) == ALIGN
        assert call("kvp_append", **{x: rows(30, 8)}) == INVAL
    assert call("kvp_append", heads=-1) == INVAL
    assert call("kvp_append", rule=0) == INVAL  # q without a rule


def test_refused_attention():
    for want, kw in ((INVAL, dict(heads=0)), (INVAL, dict(heads=6)), (INVAL, dict(window=-1)), (INVAL, dict(scale=float("nan"))), (INVAL, dict(scale=3e38)),
                     (INVAL, dict(q=rows(None))), (INVAL, dict(o=0)), (INVAL, dict(workspace=0)), (ALIGN, dict(o=at(2) + 8)), (ALIGN, dict(lse=at(3) + 2)),
                     (ALIGN, dict(workspace=at(4) + 8)), (ALIGN, dict(q=rows(1, 1028))), (INVAL, dict(q=rows(1, 1016))), (SIZE, dict(o=(1 << 64) - 1024)),
                     (SIZE, dict(workspace_bytes=100))):
        assert call("kvp_attend", **kw) == want, kw
    # units that do not fit 32 bits
    assert call("kvp_attend", c=cache(columns=1 << 18, n_seq=1000), tokens=1 << 20) == UNSUP


def test_overlaps():
    big = 7 * 8 * 128 * 2
    assert call("qk_norm_rope", q_out=N.qk_rows(at(1) + big - 16, 0, 0)) == INVAL  # of the last token
    assert call("qk_norm_rope", q_out=rows(1, 2048)) == INVAL                      # the input's address, other strides
    assert call("qk_norm_rope", k_out=rows(1)) == INVAL
    assert call("qk_norm_rope", q_out=rows(3), k_out=rows(3)) == INVAL
    assert call("qk_norm_rope", q_out=N.qk_rows(at(21), 0, 0)) == INVAL
    assert call("qk_norm_rope", k_out=N.qk_rows(at(5), 0, 0)) == INVAL
    for x, i in (("k", 10), ("v", 11), ("q_out", 10), ("q", 11), ("pos", 10), ("lens", 11), ("tok0", 10)):
        assert call("kvp_append", **{x: at(i) if x in ("pos", "lens", "tok0") else rows(i)}) == INVAL, x
    assert call("kvp_append", q_out=rows(1)) == INVAL
    assert call("kvp_append", c=cache(v=at(10) + 128)) == INVAL
    assert call("kvp_append", c=cache(table=at(10) + 128)) == INVAL
    for x, i in (("o", 1), ("o", 10), ("o", 11), ("o", 12), ("o", 13), ("lse", 2), ("lse", 14), ("workspace", 1), ("workspace", 2), ("workspace", 3)):
        assert call("kvp_attend", **{x: at(i)}) == INVAL, (x, i)


def test_heads_in_turn_that_overlap():
    # q and k of a projection [tokens, heads, (q, k, v, 16 more), d], in place; k begins inside q's heads, or q's inside k's
    def heads(i, at_channel, token=8 * 400, head=400):
        return N.qk_rows(at(i) + 2 * at_channel, token, head)

    for first, second in ((0, 120), (0, 288), (136, 16), (128, 8)):
        q, k = heads(1, first), heads(1, second)
        assert call("qk_norm_rope", q=q, q_out=q, k=k, k_out=k, kv_heads=8) == INVAL, (first, second)
    q = heads(1, 0)
    assert call("qk_norm_rope", q=q, q_out=q, k=heads(1, 128, 8 * 400, 256), k_out=rows(4)) == INVAL   # other steps


def sizes(c=None, **kw):
    c = cache() if c is None else c
    a = N.kvp_attend_args(**{**dict(cache=ct.addressof(c), tokens=7, heads=8), **kw})
    return cap.load().kvp_attend_workspace_bytes(ct.byref(a))


def test_workspace():
    assert sizes(cache(columns=8)) == 0  # 512 rows: one launch
    assert sizes() > 0 and sizes() % 8 == 0
    assert sizes(cache(columns=1 << 15)) <= (2 * 2048 * 16 * 130 * 4) + 7 * 8 * 8
    assert sizes(heads=6) == 0 and sizes(cache(d=80)) == 0 and sizes(tokens=0) == 0
    assert cap.load().kvp_attend_workspace_bytes(None) == 0
    for d in (64, 128, 256):  # that of no window does for any
        for columns in (9, 100, 5000):
            for n_seq in (1, 3, 64):
                for n in (1, 64, 500):
                    c = cache(d=d, columns=columns, n_seq=n_seq)
                    assert all(sizes(c, tokens=n, window=w) <= sizes(c, tokens=n) for w in (1, 100, 1000, 1 << 20))


def test_largest_sizes():
    # units that segments may see: below 2^31, by the table's width, or a window's
    wide = lambda columns: cache(n_seq=1024, kv_heads=8, d=64, columns=columns)
    assert sizes(wide(1 << 16), tokens=1024) > 0 == sizes(wide(1 << 18), tokens=1024)
    assert sizes(wide(1 << 18), tokens=1024, window=4000) > 0
    one = lambda columns: cache(n_seq=1, kv_heads=8, columns=columns)
    assert sizes(one(1 << 13), tokens=131072, heads=64) > 0 == sizes(one(1 << 15), tokens=131072, heads=64)
    most = (2 ** 31 - 1) // 3 // 8
    assert sizes(tokens=most) > 0 == sizes(tokens=most + 1)
    assert call("kvp_append", tokens=most + 1) == UNSUP


def test_frequencies():
    f = cap.qk_freqs(1e6, 64)
    assert f.shape == (1, 32) and f.dtype == torch.float64
    assert np.allclose(f[0].numpy(), 1e6 ** (-np.arange(32) / 32), rtol=1e-14)
    f = cap.qk_freqs(1e4, 128, sections=[16, 24, 24])
    assert [(f[a] != 0).nonzero().flatten().tolist() for a in range(3)] == [list(range(16)), list(range(16, 40)), list(range(40, 64))]
    assert torch.equal(f.sum(0), cap.qk_freqs(1e4, 128)[0])
    f = cap.qk_freqs(1e4, 32, sections=[10, 3, 3], interleave=True)
    assert [(f[a] != 0).nonzero().flatten().tolist() for a in range(3)] == [[0, 3, 6, 9, 10, 11, 12, 13, 14, 15], [1, 4, 7], [2, 5, 8]]
    f = cap.qk_freqs(1e4, 16, sections=[0, 8], interleave=True)
    assert not f[0].any() and (f[1] != 0).all()
    for kw in (dict(base=0.0, rot=64), dict(base=float("inf"), rot=64), dict(base=1e4, rot=0), dict(base=1e4, rot=64, sections=[16, 15]),
               dict(base=1e4, rot=64, sections=[33, -1])):
        with pytest.raises(cap.CapsuleError):
            cap.qk_freqs(**kw)


def test_numbers_that_no_field_holds():
    held = cache()
    handle = N.KvpCache(held, (), torch.zeros(1))
    for tokens, heads, window in ((7, 8, 1 << 31), (7, 1 << 31, 0), (1 << 63, 8, 0), (7, 8, 1.5), (7, 8, None)):
        with pytest.raises(ValueError, match="kvp_attend: .*window"):
            cap.kvp_attend_workspace_bytes(handle, tokens, heads, window)
    assert cap.kvp_attend_workspace_bytes(handle, 7, 8, (1 << 31) - 1) > 0


def test_dimensions_of_one_have_no_stride():
    # pages [kv_heads, page, d] of one head, and pools of one page out of different tensors, are refused only for not being on a GPU
    table = torch.zeros(1, 2, dtype=torch.int32)
    heads_first = torch.zeros(3, 1, 16, 64, dtype=torch.bfloat16).transpose(1, 2)
    one, other = torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16)[:1], torch.zeros(2, 3, 16, 2, 64, dtype=torch.bfloat16)[:1, 1]
    for k, v in ((heads_first, heads_first), (heads_first, torch.zeros(3, 16, 1, 64, dtype=torch.bfloat16)), (one, other)):
        with pytest.raises(ValueError, match="on one GPU"):
            cap.kvp_cache(k, v, table)


def test_binding_refuses():
    bf16, i32 = torch.bfloat16, torch.int32
    with pytest.raises(ValueError, match="on one GPU"):
        cap.qk_rule(torch.zeros(1, 8, dtype=torch.float64), eps=1e-6)
    with pytest.raises(ValueError, match="on one GPU"):
        cap.kvp_cache(torch.zeros(2, 16, 1, 64, dtype=bf16), torch.zeros(2, 16, 1, 64, dtype=bf16), torch.zeros(1, 2, dtype=i32))
    pool = torch.zeros(2, 16, 2, 64, dtype=bf16)
    for k, v, t in ((pool[0], pool, 0), (pool.float(), pool, 0), (pool.transpose(1, 2), pool, 0), (pool, pool[:1], 0),
                    (pool[:1].expand(2, -1, -1, -1), pool, 0), (pool[..., :32], pool[..., :32], 0)):
        with pytest.raises(ValueError, match="pages are contiguous"):
            cap.kvp_cache(k, v, torch.zeros(1, 2, dtype=i32))
    for t in (torch.zeros(2, dtype=i32), torch.zeros(1, 2, dtype=torch.int64), torch.zeros(2, 4, dtype=i32)[:, ::2], torch.zeros(1, 2, dtype=i32).expand(2, 2)):
        with pytest.raises(ValueError, match="table"):
            cap.kvp_cache(pool, pool, t)
    plain = cap.qk_rule(eps=1e-6)
    x = torch.zeros(3, 2, 64)
    with pytest.raises(ValueError, match="current GPU"):
        cap.qk_norm_rope(plain, x, x.clone())
    with pytest.raises(ValueError, match="neither"):
        cap.qk_norm_rope(plain, None, None)
    with pytest.raises(ValueError, match="without q"):
        cap.qk_norm_rope(plain, None, x, q_out=x)
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        cap.qk_norm_rope(plain, x.half(), x)
    with pytest.raises(ValueError, match="of shape"):
        cap.qk_norm_rope(plain, x, x, q_out=x[:2])
    with pytest.raises(ValueError, match="of shape"):
        cap.qk_norm_rope(plain, x, x.bfloat16())
    with pytest.raises(ValueError, match="overlap"):
        cap.qk_norm_rope(plain, x[:1].expand(3, 2, 64), x)
    with pytest.raises(ValueError, match="overlap"):
        cap.qk_norm_rope(plain, torch.zeros(3, 64, 2).transpose(1, 2), x)
    with pytest.raises(ValueError, match="without a norm"):
        cap.qk_rule(wq=torch.zeros(64))
