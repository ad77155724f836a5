"""Refusals of the block-scaled FP8 KV cache calls, on the host: the status codes of the C ABI with addresses that are
never used, and what the binding refuses by itself."""
import ctypes as ct

import numpy as np
import pytest
import torch

import paper_2606_20537_amd as cap
from paper_2606_20537_amd import _native as N

A = 1 << 40  # addresses far apart; nothing reads them


def seq(i=0, **kw):
    f = dict(k=A + (i << 36), v=A + (i << 36) + (1 << 34), scales=A + (i << 36) + (2 << 34), bounds=A + (i << 36) + (3 << 34),
             open=A + (i << 36) + (3 << 34) + (1 << 33), rows=1024, n=100, T=3)
    return {**f, **kw}


def table(*seqs):
    arr = (N.kvb_seq * max(1, len(seqs)))()
    for i, s in enumerate(seqs):
        arr[i] = N.kvb_seq(*[s[k] for k in ("k", "v", "scales", "bounds", "open", "rows", "n", "T")])
    return arr


def call(name, seqs=None, **kw):
    seqs = [seq()] if seqs is None else seqs
    arr = table(*seqs)
    B = 1 << 50
    f = dict(seqs=ct.addressof(arr), tokens=sum(s["T"] for s in seqs), n_seq=len(seqs), kv_heads=4, d=128, in_dtype=cap.CAP_DTYPE_BF16)
    if name == "kvb_append":
        f.update(k=B, v=B + (1 << 40), k_stride=0, v_stride=0)
        args = N.kvb_append_args
    else:
        f.update(q=B, workspace=B + (2 << 40), workspace_bytes=1 << 30, q_stride=0, heads=8)
        if name == "kvb_attend":
            f.update(o=B + (1 << 40), lse=B + (3 << 40), idx=0, n_sel=0, scale=1.0, reserved=0)
            args = N.kvb_attend_args
        else:
            f.update(idx=B + (1 << 40), n_sel=8, first=1, last=2)
            args = N.kvb_select_args
    f["seqs"] = kw.pop("address", f["seqs"])
    f.update(kw)
    a = args(**f)
    return getattr(cap.load(), name)(ct.byref(a), None)


ALL = ["kvb_append", "kvb_attend", "kvb_select"]


@pytest.mark.parametrize("name", ALL)
@pytest.mark.parametrize("want, kw", [
    (cap.CAP_E_INVAL, dict(address=0)), (cap.CAP_E_INVAL, dict(n_seq=-1)), (cap.CAP_E_INVAL, dict(kv_heads=0)), (cap.CAP_E_INVAL, dict(d=0)),
    (cap.CAP_E_INVAL, dict(tokens=4)), (cap.CAP_E_INVAL, dict(tokens=-3)), (cap.CAP_E_INVAL, dict(in_dtype=7)),
    (cap.CAP_E_UNSUPPORTED, dict(in_dtype=cap.CAP_DTYPE_F32)), (cap.CAP_E_UNSUPPORTED, dict(d=96)), (cap.CAP_E_UNSUPPORTED, dict(d=512)),
    (cap.CAP_E_UNSUPPORTED, dict(kv_heads=1 << 20, heads=1 << 20, d=256)),
])
def test_shared_refusals(name, want, kw):
    if name == "kvb_append":
        kw = {k: v for k, v in kw.items() if k != "heads"}
    assert call(name, **kw) == want


@pytest.mark.parametrize("name", ALL)
@pytest.mark.parametrize("want, s", [
    (cap.CAP_E_INVAL, dict(rows=1000)), (cap.CAP_E_INVAL, dict(rows=-64)), (cap.CAP_E_INVAL, dict(n=-1, T=0)),
    (cap.CAP_E_INVAL, dict(T=-1)), (cap.CAP_E_INVAL, dict(n=2, T=3)), (cap.CAP_E_SIZE, dict(n=1025)),
    (cap.CAP_E_UNSUPPORTED, dict(rows=(1 << 31) + 64)), (cap.CAP_E_INVAL, dict(scales=0)), (cap.CAP_E_ALIGN, dict(scales=A + 2)),
    (cap.CAP_E_ALIGN, dict(bounds=A + (3 << 34) + 8)),
])
def test_refused_sequences(name, want, s):
    assert call(name, [seq(), seq(1, **s)]) == want


def test_missing_parts():
    for part in ("k", "v", "open"):
        assert call("kvb_append", [seq(**{part: 0})]) == cap.CAP_E_INVAL
    for part in ("k", "v"):
        assert call("kvb_attend", [seq(**{part: 0})]) == cap.CAP_E_INVAL
    assert call("kvb_select", [seq(bounds=0)]) == cap.CAP_E_INVAL
    for name, args in (("kvb_append", "kv"), ("kvb_attend", "qo"), ("kvb_select", "q")):
        for x in args:
            assert call(name, **{x: 0}) == cap.CAP_E_INVAL
    assert call("kvb_select", idx=0) == cap.CAP_E_INVAL
    for name in ALL:
        assert getattr(cap.load(), name)(None, None) == cap.CAP_E_INVAL


def test_too_many_sequences():
    for name in ALL:
        assert call(name, [seq(i) for i in range(cap.KVB_MAX_SEQ + 1)]) == cap.CAP_E_UNSUPPORTED


@pytest.mark.parametrize("name", ALL)
def test_nothing_to_do(name):
    assert call(name, []) == cap.CAP_OK
    assert call(name, [seq(T=0), seq(1, T=0, n=0, rows=0, k=0, v=0, scales=0, bounds=0, open=0)]) == cap.CAP_OK


@pytest.mark.parametrize("name, field", [("kvb_append", "k_stride"), ("kvb_append", "v_stride"), ("kvb_attend", "q_stride"), ("kvb_select", "q_stride")])
def test_strides(name, field):
    width = 512 if name == "kvb_append" else 1024
    assert call(name, **{field: width - 8}) == cap.CAP_E_INVAL
    assert call(name, **{field: -width}) == cap.CAP_E_INVAL
    assert call(name, **{field: width + 4}) == cap.CAP_E_ALIGN
    assert call(name, **{field: (1 << 30) + 8}) == cap.CAP_E_UNSUPPORTED


def test_alignment():
    for name, fields in (("kvb_append", "kv"), ("kvb_attend", ["q", "o"]), ("kvb_select", ["q", "workspace"])):
        for x in fields:
            assert call(name, **{x: (1 << 50) + 8}) == cap.CAP_E_ALIGN
    assert call("kvb_attend", lse=(1 << 50) + (1 << 45) + 2) == cap.CAP_E_ALIGN
    assert call("kvb_attend", idx=(1 << 50) + (1 << 45) + 1, n_sel=4) == cap.CAP_E_ALIGN


def test_overlaps():
    s = seq()
    for part in ("k", "v", "scales", "bounds", "open"):
        assert call("kvb_append", k=s[part] + 64) == cap.CAP_E_INVAL
        assert call("kvb_append", [s, seq(1, **{part: s[part] + (0 if part == "scales" else 64)})]) == cap.CAP_E_INVAL
    assert call("kvb_append", [s, s]) == cap.CAP_E_INVAL
    q = 1 << 50
    for kw in (dict(o=q), dict(lse=q), dict(o=s["k"]), dict(lse=s["scales"]), dict(o=q + (1 << 40), lse=q + (1 << 40)),
               dict(idx=q + (1 << 40), n_sel=4)):
        assert call("kvb_attend", **kw) == cap.CAP_E_INVAL
    big = [seq(rows=1 << 16, n=1 << 16)]
    assert call("kvb_attend", big, workspace=q) == cap.CAP_E_INVAL
    for kw in (dict(idx=q), dict(workspace=q), dict(idx=s["bounds"]), dict(workspace=s["scales"])):
        assert call("kvb_select", **kw) == cap.CAP_E_INVAL


def test_attend_own_refusals():
    assert call("kvb_attend", heads=6) == cap.CAP_E_INVAL
    assert call("kvb_attend", heads=0) == cap.CAP_E_INVAL
    assert call("kvb_attend", n_sel=4) == cap.CAP_E_INVAL
    assert call("kvb_attend", idx=(1 << 50) + (1 << 45), n_sel=0) == cap.CAP_E_INVAL
    assert call("kvb_attend", reserved=1) == cap.CAP_E_INVAL
    for scale in (float("nan"), float("inf")):
        assert call("kvb_attend", scale=scale) == cap.CAP_E_INVAL
    assert call("kvb_attend", [seq(rows=1 << 16, n=1 << 16)], workspace_bytes=16) == cap.CAP_E_SIZE
    assert call("kvb_attend", [seq(rows=1 << 16, n=1 << 16)], workspace=0, workspace_bytes=0) == cap.CAP_E_INVAL


def test_select_own_refusals():
    for kw in (dict(first=-1), dict(last=0), dict(n_sel=0), dict(n_sel=2), dict(first=7), dict(first=(1 << 31) - 1, last=(1 << 31) - 1)):
        assert call("kvb_select", **kw) == cap.CAP_E_INVAL
    assert call("kvb_select", workspace_bytes=8) == cap.CAP_E_SIZE
    assert call("kvb_select", workspace=0) == cap.CAP_E_INVAL


def test_workspace_sizes():
    lib = cap.load()
    arr = table(seq(), seq(1, T=0), seq(2, n=65, T=1))
    a = N.kvb_select_args(seqs=ct.addressof(arr), tokens=4, n_seq=3, heads=8, kv_heads=4, d=128, n_sel=8, first=1, last=2, in_dtype=cap.CAP_DTYPE_BF16)
    assert lib.kvb_select_workspace_bytes(ct.byref(a)) == (3 * 4 * 2 + 1 * 4 * 2) * 8
    a.d = 100
    assert lib.kvb_select_workspace_bytes(ct.byref(a)) == 0
    assert lib.kvb_select_workspace_bytes(None) == 0 and lib.kvb_attend_workspace_bytes(None) == 0
    arr = table(seq(n=64, T=1))
    a = N.kvb_attend_args(seqs=ct.addressof(arr), tokens=1, n_seq=1, heads=8, kv_heads=4, d=128, in_dtype=cap.CAP_DTYPE_BF16)
    assert lib.kvb_attend_workspace_bytes(ct.byref(a)) == 0  # one block: one run
    arr[0].rows = arr[0].n = 1 << 20
    need = lib.kvb_attend_workspace_bytes(ct.byref(a))
    assert 0 < need <= 64 << 20 and need % 16 == 0
    a.tokens = 2
    assert lib.kvb_attend_workspace_bytes(ct.byref(a)) == 0


def test_binding_refusals():
    t = cap.kvb_seqs([[0, 0, 0, 0, 0, 64, 3, 3]])
    k = torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    o, idx = torch.zeros((3, 4, 64), dtype=torch.bfloat16), torch.zeros((3, 2, 4), dtype=torch.int32)
    q = torch.zeros((3, 4, 64), dtype=torch.bfloat16)
    for bad in (t.astype(np.int32), t[:, :7], t.reshape(-1), np.asfortranarray(np.concatenate([t, t]))):
        with pytest.raises(ValueError):
            cap.kvb_append(bad, k, k, stream=0)
    for bad in (k.half(), k[0], k.transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises(ValueError):
            cap.kvb_append(t, bad, k, stream=0)
    for bad in (k[:2], k.float()):
        with pytest.raises(ValueError):
            cap.kvb_append(t, k, bad, stream=0)
    for kw in (dict(o=o[:2]), dict(o=o.float()), dict(lse=torch.zeros(3, 4, dtype=torch.bfloat16)), dict(lse=torch.zeros(4, 3).t()), dict(idx=idx.long()),
               dict(idx=idx[:, :1])):
        with pytest.raises(ValueError):
            cap.kvb_attend(t, q, **{"o": o, "kv_heads": 2, "scale": 1.0, "stream": 0, **kw})
    for bad in (idx.long(), idx[:2], torch.zeros((2, 3, 4), dtype=torch.int32).transpose(0, 1)):
        with pytest.raises(ValueError):
            cap.kvb_select(t, q, bad, kv_heads=2, stream=0)
    for call_ in (lambda: cap.kvb_append(t, k, k, stream=0), lambda: cap.kvb_attend(t, q, o, kv_heads=2, scale=1.0, stream=0),
                  lambda: cap.kvb_select(t, q, idx, kv_heads=2, stream=0)):
        with pytest.raises(ValueError, match="GPU"):  # host tensors
            call_()
    assert cap.kvb_seqs([]).shape == (0, 8)


def test_plain_forms():
    """The plain encoder against torch's conversion, at every code and between any two."""
    import kvb_plain as P
    v = np.sort(P.CODES[~np.isnan(P.CODES)])
    mid = (v[1:] + v[:-1]) / 2
    x = np.concatenate([v, mid, np.nextafter(mid, np.inf), np.nextafter(mid, -np.inf)])
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).double().numpy()
    same = torch.from_numpy(x).float().double().numpy() == x  # (neighbours that fp32 cannot hold are skipped)
    assert np.array_equal(P.nearest(x)[same], want[same])
    for amax in (0.0, 1e-40, 448.0, 448.001, 3e38, 7.5, 896.0):
        e = P.exponent(amax)
        assert e in (-100, 119) or 448.0 * 2.0 ** (e - 1) < amax <= 448.0 * 2.0 ** e


def test_binding_refuses_tokens_that_overlap():
    """One row broadcast over the tokens has a stride of zero, which the library takes for contiguous; rows that share
    elements have one below a row."""
    t = cap.kvb_seqs([[0, 0, 0, 0, 0, 64, 3, 3]])
    k, q = torch.zeros((3, 2, 64), dtype=torch.bfloat16), torch.zeros((3, 4, 64), dtype=torch.bfloat16)
    idx = torch.zeros((3, 2, 4), dtype=torch.int32)
    flat = torch.zeros(1024, dtype=torch.bfloat16)
    for bad in (k[:1].expand(3, 2, 64), flat.as_strided((3, 2, 64), (64, 64, 1))):
        for args in ((bad, k), (k, bad)):
            with pytest.raises(ValueError, match="overlap"):
                cap.kvb_append(t, *args, stream=0)
    for bad in (q[:1].expand(3, 4, 64), flat.as_strided((3, 4, 64), (8, 64, 1))):
        with pytest.raises(ValueError, match="overlap"):
            cap.kvb_attend(t, bad, torch.empty_like(q), kv_heads=2, scale=1.0, stream=0)
        with pytest.raises(ValueError, match="overlap"):
            cap.kvb_select(t, bad, idx, kv_heads=2, stream=0)
    # a single token broadcast over one is one token
    assert N._kvb_tokens("kvb_append", "k", k[:1].expand(1, 2, 64))[0] == 0
    assert N._kvb_tokens("kvb_append", "k", torch.zeros((3, 5, 64), dtype=torch.bfloat16)[:, 1:3])[0] == 320


def test_binding_refuses_a_workspace_that_is_not_contiguous(monkeypatch):
    """A view's elements are not the bytes behind its address: 64 elements of one broadcast byte, every other byte."""
    monkeypatch.setattr(N, "_kvb_device", lambda *a: None)
    t = cap.kvb_seqs([[0, 0, 0, 0, 0, 64, 3, 3]])  # (no addresses: the library refuses the call behind the check)
    q, idx = torch.zeros((3, 4, 64), dtype=torch.bfloat16), torch.zeros((3, 2, 4), dtype=torch.int32)
    ws = torch.zeros(4096, dtype=torch.uint8)
    for bad in (ws[:1].expand(4096), ws[::2], ws.view(64, 64).t()):
        with pytest.raises(ValueError, match="contiguous"):
            cap.kvb_attend(t, q, torch.empty_like(q), kv_heads=2, scale=1.0, workspace=bad, stream=0)
        with pytest.raises(ValueError, match="contiguous"):
            cap.kvb_select(t, q, idx, kv_heads=2, workspace=bad, stream=0)


def test_sequence_table_refuses_buffers_that_are_not_contiguous():
    """One layer's rows out of a buffer of several layers: the library would read the other layers' as the next rows."""
    k = torch.zeros((128, 2, 64), dtype=torch.uint8)
    scales, bounds = torch.zeros((2, 2, 2)), torch.zeros((2, 2, 2, 64), dtype=torch.uint8)
    open_ = torch.zeros((2, 64, 2, 64), dtype=torch.bfloat16)
    good = [k, k.clone(), scales, bounds, open_]
    assert cap.kvb_seqs([(*good, 128, 3, 3)])[0].tolist() == [x.data_ptr() for x in good] + [128, 3, 3]
    for i, x in enumerate(good):
        layers = torch.zeros((x.shape[0], 4, *x.shape[1:]), dtype=x.dtype)
        with pytest.raises(ValueError, match="contiguous"):
            cap.kvb_seqs([(*good, 128, 3, 3), (*good[:i], layers[:, 1], *good[i + 1:], 128, 3, 3)])


def test_binding_takes_a_single_head_of_any_stride():
    """One head of a token has no neighbour: every fifth of five, or the last, with the stride of the tokens alone."""
    x = torch.zeros((3, 5, 64), dtype=torch.bfloat16)
    for one in (x[:, ::5], x.transpose(0, 1).contiguous().transpose(0, 1)[:, 4:], x.as_strided((3, 1, 64), (320, 7, 1))):
        assert N._kvb_tokens("kvb_append", "k", one)[0] == (one.stride(0) if not one.is_contiguous() else 0)


def test_attend_refuses_a_scale_whose_multiple_of_log2_e_is_not_finite():
    """Scores are held in units of log 2: 3e38 log2(e) would be infinite, and times a score of zero NaN."""
    for scale in (3e38, -3e38, 2.4e38):
        assert call("kvb_attend", scale=scale) == cap.CAP_E_INVAL


def test_buffers_that_end_past_the_last_address():
    """An end that wraps round to a small address would overlap nothing."""
    end = (1 << 64) - 256
    for part in ("k", "v", "scales", "bounds", "open"):
        assert call("kvb_append", [seq(**{part: end})]) == cap.CAP_E_SIZE
    for part in ("k", "v", "scales"):
        assert call("kvb_attend", [seq(**{part: end})]) == cap.CAP_E_SIZE
    for part in ("scales", "bounds"):
        assert call("kvb_select", [seq(**{part: end})]) == cap.CAP_E_SIZE
    wide = dict(k_stride=1 << 20, v_stride=1 << 20)
    for x in ("k", "v"):
        assert call("kvb_append", **{x: end, **wide}) == cap.CAP_E_SIZE
    big = [seq(rows=1 << 16, n=1 << 16)]
    for x in ("q", "o", "lse", "workspace"):
        assert call("kvb_attend", big, **{x: end if x != "lse" else (1 << 64) - 16, "q_stride": 1 << 20}) == cap.CAP_E_SIZE
    assert call("kvb_attend", idx=(1 << 64) - 16, n_sel=4) == cap.CAP_E_SIZE
    for x in ("q", "idx", "workspace"):
        assert call("kvb_select", big, **{x: end if x == "q" else (1 << 64) - 16, "q_stride": 1 << 20}) == cap.CAP_E_SIZE


@pytest.mark.parametrize("d", [64, 128, 256])
def test_attend_workspace_is_bounded(d):
    """Whatever the batch: 1024 parts of 128 rows, and as many of 16 (runs of a 512th of their blocks and more, of which a
    cut sequence's last may be short)."""
    most = (1024 * 128 + 1024 * 16) * (d + 2) * 4
    rng = np.random.default_rng(4)
    for _ in range(300):
        seqs = []
        for i in range(rng.integers(1, 9)):
            T = int(2 ** rng.uniform(0, 12)) if rng.random() < 0.6 else 1
            n = T + int(2 ** rng.uniform(0, 17))
            seqs.append(seq(i, n=n, T=T, rows=-(-n // 64) * 64))
        arr = table(*seqs)
        hkv = int(rng.choice([1, 2, 4, 8]))
        a = N.kvb_attend_args(seqs=ct.addressof(arr), tokens=sum(s["T"] for s in seqs), n_seq=len(seqs), heads=hkv * int(rng.choice([1, 4, 8])),
                              kv_heads=hkv, d=d, in_dtype=cap.CAP_DTYPE_BF16)
        assert cap.load().kvb_attend_workspace_bytes(ct.byref(a)) <= most
