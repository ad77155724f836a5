"""Norm and rotation of q and k against their 64-bit plain form, in place, strided and under capture."""
import numpy as np
import pytest
import torch

import kvp_plain as plain
import paper_2606_20537_amd as cap

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def host(x):
    return x.detach().cpu().double().numpy()


def normal(seed, *shape):
    return torch.randn(shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")


def positions(seed, tokens, axes, top):
    return torch.randint(0, top, (tokens, axes), generator=torch.Generator("cuda").manual_seed(seed), device="cuda", dtype=torch.int32)


def check(got, x, w, pos, freqs, eps, w_add, rot, pairs):
    want, size = plain.turned(host(x), None if w is None else host(w), None if pos is None else pos.cpu().numpy(), None if freqs is None else host(freqs),
                              eps, w_add, rot, pairs)
    assert plain.turned_near(host(got), want, size, HALF[got.dtype])


def freqs_of(rot, axes, base=1e6):
    return cap.qk_freqs(base, rot, None if axes == 1 else [rot // 2 - (axes - 1) * (rot // 2 // axes)] + [rot // 2 // axes] * (axes - 1), True).cuda()


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d, rot", [(16, 16), (16, 0), (48, 16), (64, 64), (80, 80), (96, 32), (128, 128), (192, 64), (256, 64), (256, 256), (512, 512), (512, 16)])
def test_channels(d, rot, dtype, pairs):
    tokens, heads, kv = 5, 3, 2
    q, k = (3.0 * normal(d + rot + i, tokens, h, d).to(dtype) for i, h in enumerate((heads, kv)))
    wq, wk = (1 + 0.3 * normal(7 + i, d).to(dtype) for i in range(2))
    f = freqs_of(rot, 1) if rot else None
    pos = positions(3, tokens, 1, 1 << 17) if rot else None
    for eps, wa, wb, w_add in ((1e-6, wq, wk, 0.0), (1e-5, wq, None, 1.0), (None, None, None, 0.0)):
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        cap.qk_norm_rope(cap.qk_rule(f, wq=wa, wk=wb, eps=eps, w_add=w_add, pairs=pairs), q, k, qo, ko, pos=pos)
        check(qo, q, wa, pos, f, eps, w_add, rot, pairs)
        check(ko, k, wb, pos, f, eps, w_add, rot, pairs)


@pytest.mark.parametrize("tokens", [1, 2, 511, 513, 1024, 4097])
@pytest.mark.parametrize("heads, kv, axes", [(1, 1, 1), (5, 0, 2), (0, 3, 3), (32, 4, 8)])
def test_counts(tokens, heads, kv, axes):
    d, rot = 64, 32
    q, k = (normal(tokens + i, tokens, h, d).bfloat16() if h else None for i, h in enumerate((heads, kv)))
    w = (1 + 0.3 * normal(7, d))
    f, pos = freqs_of(rot, axes), positions(3, tokens, axes, 1000)
    qo, ko = (torch.empty_like(x) if x is not None else None for x in (q, k))
    cap.qk_norm_rope(cap.qk_rule(f, wq=w, wk=w, eps=1e-6), q, k, qo, ko, pos=pos)  # float32 weights beside bfloat16 rows
    for got, x in ((qo, q), (ko, k)):
        if x is not None:
            check(got, x, w, pos, f, 1e-6, 0.0, rot, False)


@pytest.mark.parametrize("pos", [[0, 1, -1, -77], [1 << 20, (1 << 24) + 1, (1 << 30) + 3, (1 << 31) - 1]])
def test_far_positions(pos):
    pos = torch.tensor(pos, dtype=torch.int32, device="cuda")
    q = normal(1, 4, 2, 64)
    f = freqs_of(64, 1)
    out = torch.empty_like(q)
    cap.qk_norm_rope(cap.qk_rule(f), q, None, out, pos=pos)
    check(out, q, None, pos[:, None], f, None, 0.0, 64, False)


def test_axes_add_up():
    # every axis turns every pair
    f = torch.stack([cap.qk_freqs(b, 32)[0] for b in (1e2, 1e4, 1e6)]).cuda()
    q, pos = normal(1, 50, 2, 32), positions(2, 50, 3, 5000)
    out = torch.empty_like(q)
    cap.qk_norm_rope(cap.qk_rule(f, pairs=True), q, None, out, pos=pos)
    check(out, q, None, pos, f, None, 0.0, 32, True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_slices_of_a_projection_in_place(dtype):
    # [query head, gate] by query head, then K, then V
    tokens, heads, kv, d = 67, 5, 2, 64
    x = normal(4, tokens, 2 * heads + 2 * kv, d).to(dtype)
    before = x.clone()
    q, k = x[:, :2 * heads:2], x[:, 2 * heads:2 * heads + kv]
    f, pos, w = freqs_of(64, 1), positions(3, tokens, 1, 4096), (1 + 0.2 * normal(8, d)).to(dtype)
    rule = cap.qk_rule(f, wq=w, wk=w, eps=1e-6)
    qo, ko = torch.empty((tokens, heads, d), dtype=dtype, device="cuda"), torch.empty((tokens, kv, d), dtype=dtype, device="cuda")
    cap.qk_norm_rope(rule, q, k, qo, ko, pos=pos)
    assert torch.equal(x, before)
    check(qo, q, w, pos, f, 1e-6, 0.0, 64, False)
    check(ko, k, w, pos, f, 1e-6, 0.0, 64, False)
    cap.qk_norm_rope(rule, q, k, pos=pos)
    assert torch.equal(q, qo) and torch.equal(k, ko)
    assert torch.equal(x[:, 1:2 * heads:2], before[:, 1:2 * heads:2]) and torch.equal(x[:, 2 * heads + kv:], before[:, 2 * heads + kv:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ends_of_the_range(dtype):
    # squares that overflow and that vanish, zeros; the norm of an infinite row is 0 or NaN, and stays in its row
    d = 128
    size = torch.tensor([1e37, 2.0 ** 100, 2.0 ** 64, 1e-30, 0.0, 1.0], device="cuda")[:, None, None]
    q = (normal(5, 6, 2, d).clamp(-3, 3) * size).to(dtype)
    rule = cap.qk_rule(eps=1e-6)
    out = torch.empty_like(q)
    cap.qk_norm_rope(rule, q, None, out)
    check(out, q, None, None, None, 1e-6, 0.0, 0, False)
    q[5, 0, 3] = float("inf")
    q[4, 1, 7] = float("nan")
    again = torch.empty_like(q)
    cap.qk_norm_rope(rule, q, None, again)
    assert torch.equal(again[:4], out[:4]) and torch.equal(again[5, 1], out[5, 1]) and torch.equal(again[4, 0], out[4, 0])
    assert again[5, 0, 3].isnan() and not again[5, 0, :3].any() and again[4, 1].isnan().all()


def test_unit_length_for_the_delta_rule():
    d = 128
    w = torch.full((d,), d ** -0.5, device="cuda")
    k = normal(3, 300, 4, d)
    out = torch.empty_like(k)
    cap.qk_norm_rope(cap.qk_rule(wk=w, eps=1e-12), None, k, None, out)
    assert (out.norm(dim=-1) - 1).abs().max() < 1e-5


def test_rule_of_other_channels():
    rule = cap.qk_rule(wq=torch.ones(64, device="cuda"), eps=1e-6)
    q = normal(1, 2, 2, 128)
    with pytest.raises(ValueError, match="64 channels"):
        cap.qk_norm_rope(rule, q, None)
    f = freqs_of(128, 1)
    with pytest.raises(cap.CapsuleError):
        cap.qk_norm_rope(cap.qk_rule(f), normal(1, 2, 2, 64), None, pos=positions(1, 2, 1, 9))  # more rotated channels than there are
    with pytest.raises(cap.CapsuleError):
        cap.qk_norm_rope(cap.qk_rule(f), q, None)  # no positions
    with pytest.raises(ValueError, match="pos"):
        cap.qk_norm_rope(cap.qk_rule(f), q, None, pos=positions(1, 3, 1, 9))


def test_capture_and_streams():
    tokens, d = 40, 64
    q, k = normal(1, tokens, 4, d).bfloat16(), normal(2, tokens, 2, d).bfloat16()
    pos, f = positions(3, tokens, 1, 99), freqs_of(d, 1)
    rule = cap.qk_rule(f, eps=1e-6)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cap.qk_norm_rope(rule, q, k, qo, ko, pos=pos)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    go, gk = torch.empty_like(q), torch.empty_like(k)
    with torch.cuda.graph(g):
        cap.qk_norm_rope(rule, q, k, go, gk, pos=pos)
    for i in range(3):
        q.copy_(normal(10 + i, tokens, 4, d))
        pos += 5
        g.replay()
        cap.qk_norm_rope(rule, q, k, qo, ko, pos=pos)
        torch.cuda.synchronize()
        assert torch.equal(go, qo) and torch.equal(gk, ko)
        check(go, q, None, pos, f, 1e-6, 0.0, d, False)
