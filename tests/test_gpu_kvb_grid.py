"""Calls on the block-scaled FP8 KV cache whose launches have more than 2^24 workgroups, which a grid along x alone cannot
count (its threads are counted in 32 bits): equal to the same work in parts."""
import numpy as np
import pytest
import torch

import kvb_plain as P
import paper_2606_20537_amd as cap
from test_gpu_kvb import BLOCK, values

pytestmark = pytest.mark.gpu


def test_select_scores():
    """64 sequences of one token, 1024 KV heads, 4112 blocks: 1024 x 64 x 257 workgroups of scores."""
    n_seq, hkv, d, nb, n_sel = 64, 1024, 64, 4112, 6
    g = torch.Generator(device="cuda").manual_seed(1)
    bounds = torch.randint(0, 0x78, (nb, 2, hkv, d), generator=g, dtype=torch.uint8, device="cuda")
    bounds[:, 0] |= 0x80
    scales = torch.ones((nb, 2, hkv), device="cuda")
    q = torch.randn((n_seq, hkv, d), generator=g, device="cuda").bfloat16()
    seqs = cap.kvb_seqs([(0, 0, scales, bounds, 0, nb * BLOCK, nb * BLOCK - 3 * i, 1) for i in range(n_seq)])
    idx, parts = (torch.full((n_seq, hkv, n_sel), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    cap.kvb_select(seqs, q, idx, kv_heads=hkv, first=1, last=2)
    for i in range(0, n_seq, 16):
        cap.kvb_select(seqs[i:i + 16].copy(), q[i:i + 16], parts[i:i + 16], kv_heads=hkv, first=1, last=2)
    assert torch.equal(idx, parts)
    for i, h in ((0, 0), (31, 511), (63, 0), (63, 1023)):
        want = P.select(q[i, h:h + 1].double().cpu().numpy(), values(bounds[:, :, h]), np.ones(nb), n_sel, 1, 2, nb * BLOCK - 3 * i - 1)
        assert idx[i, h].tolist() == want


def test_choices_and_listed_blocks():
    """64 sequences of 260 tokens, 1024 KV heads: 17 million choices, and as many workgroups of attention over them."""
    n_seq, T, hkv, d, n_sel = 64, 260, 1024, 64, 2
    g = torch.Generator(device="cuda").manual_seed(2)
    rows = -(-T // BLOCK) * BLOCK
    kv, open_ = torch.zeros((2, rows, hkv, d), dtype=torch.uint8, device="cuda"), torch.zeros((2, BLOCK, hkv, d), dtype=torch.bfloat16, device="cuda")
    scales, bounds = torch.ones((rows // BLOCK, 2, hkv), device="cuda"), torch.zeros((rows // BLOCK, 2, hkv, d), dtype=torch.uint8, device="cuda")
    one = cap.kvb_seqs([(kv[0], kv[1], scales, bounds, open_, rows, T, T)])
    new = torch.randn((2, T, hkv, d), generator=g, device="cuda").bfloat16()
    cap.kvb_append(one, new[0], new[1])
    seqs = np.repeat(one, n_seq, 0)  # every sequence the same rows, queries of its own
    q = torch.randn((n_seq * T, hkv, d), generator=g, device="cuda", dtype=torch.bfloat16)
    idx = torch.full((n_seq * T, hkv, n_sel), -7, dtype=torch.int32, device="cuda")
    o = torch.full_like(q, 7.0)
    cap.kvb_select(seqs, q, idx, kv_heads=hkv, first=0, last=1)
    cap.kvb_attend(seqs, q, o, kv_heads=hkv, scale=0.125, idx=idx)
    for i in (0, 1, 62, 63):
        at = slice(i * T, (i + 1) * T)
        part, out = torch.empty_like(idx[at]), torch.empty_like(o[at])
        cap.kvb_select(one, q[at], part, kv_heads=hkv, first=0, last=1)
        cap.kvb_attend(one, q[at], out, kv_heads=hkv, scale=0.125, idx=part)
        assert torch.equal(idx[at], part) and torch.equal(o[at], out)
    assert not (idx == -7).any() and not (o == 7.0).all(-1).any()
