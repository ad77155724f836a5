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
