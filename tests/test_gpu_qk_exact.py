"""Norm and rotation of q and k where every bit counts: angles, and values that a call leaves alone."""
import numpy as np
import pytest
import torch

import paper_2606_20537_amd as cap

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("quarter", [0, 1, 2, 3])
def test_small_sines_and_cosines(quarter, pairs):
    # Angles at and near multiples of a quarter turn: the small one of the two is as near, relative to itself, as fp32 allows:
    # 4 * 2^-24 of sine and cosine, the rest's product and sum (2 * 2^-24) and two products and a sum with a row of ones and zeros (none);
    # the angle in 64 bits is off by four roundings of less than 8.
    tokens, d = 50, 128
    far = torch.linspace(-30, -6, tokens * d // 2, dtype=torch.float64).exp2().view(tokens, d // 2) * (1 - 2 * (torch.arange(d // 2) % 2))
    far[0] = 0
    for t in range(tokens):  # a table for each: one token at position 1
        f = (2 * np.pi * (quarter / 4 + far[t].numpy()))[None]
        x = torch.zeros((1, 1, d), device="cuda")
        x[..., 0::2] = 1.0
        if not pairs:
            x[..., :d // 2], x[..., d // 2:] = 1.0, 0.0
        out = torch.empty_like(x)
        cap.qk_norm_rope(cap.qk_rule(torch.from_numpy(f).cuda(), pairs=pairs), x, None, out, pos=torch.ones(1, dtype=torch.int32, device="cuda"))
        out = out.cpu().double().numpy()[0, 0]
        c, s = (out[0::2], out[1::2]) if pairs else (out[:d // 2], out[d // 2:])
        angle = f[0].astype(np.longdouble)
        for got, exact in ((c, np.cos(angle)), (s, np.sin(angle))):
            exact = exact.astype(np.float64)
            assert (np.abs(got - exact) <= 6 * 2.0 ** -24 * np.abs(exact) + 4 * 8 * 2.0 ** -53).all()


def patterns(dtype, shape):
    """Every bf16 pattern in turn, and fp32 ones whose upper halves are those."""
    n = int(np.prod(shape))
    i = torch.arange(n, dtype=torch.int64, device="cuda") % 65536
    if dtype == torch.bfloat16:
        return i.to(torch.int16).view(torch.bfloat16).view(shape)
    return ((i << 16) + (i * 40503) % 65536).to(torch.int32).view(torch.float32).view(shape)


def bits(x):
    return x.contiguous().view(torch.int16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 80, 256])
@pytest.mark.parametrize("rot, pairs", [(0, False), (0, True), (32, False), (32, True), (48, True)])
def test_channels_that_stay_keep_their_bits(dtype, d, rot, pairs):
    # signalling NaN, infinities and denormals too; a call without norm and rotation is a copy
    x = patterns(dtype, (65536 // 64, 3, d))
    pos = torch.ones(len(x), dtype=torch.int32, device="cuda") if rot else None
    out = torch.empty_like(x)
    cap.qk_norm_rope(cap.qk_rule(cap.qk_freqs(1e4, rot).cuda() if rot else None, pairs=pairs), x, None, out, pos=pos)
    assert torch.equal(bits(out[..., rot:]), bits(x[..., rot:]))


@pytest.mark.parametrize("d", [64, 128, 256])
def test_rows_appended_without_a_rule_keep_their_bits(d):
    tokens, page = 65536 * 2 // (2 * d), 16
    k = patterns(torch.bfloat16, (tokens, 2, d))
    v = k.flip(0)
    pools = torch.zeros((2, tokens // page, page, 2, d), dtype=torch.bfloat16, device="cuda")
    table = torch.arange(tokens // page, dtype=torch.int32, device="cuda")[None]
    cap.kvp_append(cap.kvp_cache(pools[0], pools[1], table), torch.tensor([tokens], dtype=torch.int32, device="cuda"), k, v,
                   tok0=torch.tensor([0, tokens], dtype=torch.int32, device="cuda"))
    assert torch.equal(bits(pools[0].flatten(0, 1)), bits(k)) and torch.equal(bits(pools[1].flatten(0, 1)), bits(v))


def test_positions_beside_a_rule_without_rotation():
    # a layer that only norms, called as those that rotate
    x = patterns(torch.bfloat16, (5, 3, 64)).nan_to_num(1.0, 1.0, 1.0)
    rule, pos = cap.qk_rule(eps=1e-6), torch.arange(5, dtype=torch.int32, device="cuda")
    want, got = torch.empty_like(x), torch.empty_like(x)
    cap.qk_norm_rope(rule, x, None, want)
    for p in (pos, pos[:, None], pos[:, None].repeat(1, 3)):
        cap.qk_norm_rope(rule, x, None, got.zero_(), pos=p)
        assert torch.equal(got, want)
    pools = torch.zeros((2, 1, 16, 3, 64), dtype=torch.bfloat16, device="cuda")
    cache = cap.kvp_cache(pools[0], pools[1], torch.zeros((1, 1), dtype=torch.int32, device="cuda"))
    lens, tok0 = (torch.tensor(i, dtype=torch.int32, device="cuda") for i in ([5], [0, 5]))
    cap.kvp_append(cache, lens, x, x, tok0=tok0, rule=rule, pos=pos)
    assert torch.equal(pools[0, 0, :5], want) and torch.equal(pools[1, 0, :5], x)


@pytest.mark.parametrize("tokens", [1, 37])
def test_heads_of_q_k_and_v_in_turn(tokens):
    # a projection [tokens, heads, (q, k, v), d] in place
    heads, d = 4, 64
    x = torch.randn((tokens, heads, 3, d), generator=torch.Generator("cuda").manual_seed(1), device="cuda").bfloat16()
    before = x.clone()
    q, k, v = (x[:, :, i] for i in range(3))
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda")
    rule = cap.qk_rule(cap.qk_freqs(1e4, d).cuda(), eps=1e-6)
    qo, ko = torch.empty((2, tokens, heads, d), dtype=torch.bfloat16, device="cuda")
    cap.qk_norm_rope(rule, q, k, qo, ko, pos=pos)
    assert torch.equal(x, before)
    cap.qk_norm_rope(rule, q, k, pos=pos)
    assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(v, before[:, :, 2])
    x.copy_(before)
    pools = torch.zeros((2, 3, 16, heads, d), dtype=torch.bfloat16, device="cuda")
    cache = cap.kvp_cache(pools[0], pools[1], torch.arange(3, dtype=torch.int32, device="cuda")[None])
    lens, tok0 = (torch.tensor(i, dtype=torch.int32, device="cuda") for i in ([tokens], [0, tokens]))
    cap.kvp_append(cache, lens, k, v, tok0=tok0, rule=rule, q=q, pos=pos)
    assert torch.equal(q, qo) and torch.equal(x[:, :, 1:], before[:, :, 1:])
    assert torch.equal(pools[0].flatten(0, 1)[:tokens], ko) and torch.equal(pools[1].flatten(0, 1)[:tokens], v)
