"""Plain forms of the norm and rotation of q and k and of attention over a paged cache, in 64 bits on the host, and how
near the kernels' arithmetic has to come to them."""
import numpy as np


def turned(x, w, pos, freqs, eps, w_add, rot, pairs):
    """Rows x [tokens, heads, d], pos [tokens, axes], freqs [axes, rot / 2]; eps None: no norm.  Also, for each value,
    the magnitude that its errors are relative to."""
    y = np.asarray(x, np.float64)
    if eps is not None:
        f = 1.0 / np.sqrt((y * y).mean(-1, keepdims=True) + eps)
        y = y * f * (1.0 if w is None else w_add + np.asarray(w, np.float64))
    size = np.abs(y)
    if rot:
        i = np.arange(rot // 2)
        a, b = (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)
        # (an extended mantissa, as the product alone loses 2^-22 at position 2^31)
        angle = (np.asarray(pos, np.longdouble)[:, :, None] * np.asarray(freqs, np.longdouble)).sum(1)[:, None]
        c, s = np.cos(angle).astype(np.float64), np.sin(angle).astype(np.float64)
        ya, yb = y[..., a].copy(), y[..., b].copy()
        y[..., a], y[..., b] = ya * c - yb * s, yb * c + ya * s
        size[..., a] = size[..., b] = np.abs(ya) + np.abs(yb)
    return y, size


def turned_near(got, want, size, half_step):
    """Whether the kernel's values are as near as its arithmetic allows.

    Norm in fp32: a sum of squares over 16 values and 5 lanes' steps (21 roundings), its mean, eps, root and reciprocal
    (8 more halved by the root), the products with the factor and the weight, its sum with w_add (3): below 32 * 2^-24 =
    2^-19.  Angle: 2^-20 from 64 bits, its rounding in half turns pi 2^-25, sine and cosine 4 * 2^-24: below 2^-19.  Two
    products and a sum: 3 * 2^-24.  Together below 2^-17.9 of |a| + |b|; then the output's rounding."""
    far = size * 2.0 ** -17.9
    return (np.abs(got - want) <= far + (np.abs(want) + far) * half_step + 1e-40).all()


def seen_rows(pos, window, there):
    """Rows that the token at row pos sees; there[r]: row r lies on a page."""
    r = np.arange(max(0, pos - window + 1) if window else 0, min(pos + 1, len(there)))
    return r[there[r]] if len(r) else r


def attend(q, k, v, scale, rows):
    """One query row over the rows of k, v [n, d]: (o, lse, sum of weight times |v|, sum of the products' magnitudes of a
    score)."""
    d = k.shape[1]
    if len(rows) == 0:
        return np.zeros(d), -np.inf, np.zeros(d), 0.0
    k, v = k[rows], v[rows]
    with np.errstate(invalid="ignore", over="ignore"):
        x = scale * (k @ q)
        m = x.max()
        p = np.exp(x - m)
        z = p.sum()
        p = p / z
        return p @ v, m + np.log(z), p @ np.abs(v), np.abs(scale * k * q).sum(1).max()


def attend_near(o, lse, plain, n):
    """Whether a row's results are as near as the arithmetic allows.

    Scores: sums of d <= 256 products in fp32 (256 * 2^-24 of their magnitudes), times the scale; exponents in fp32
    (2^-22 of score and reference, which stands 32 above a score).  A score's error dx changes a weight by the factor 1 +- 2 dx (weight and sum).
    Weights enter as hi + lo, two bf16 (2^-16), sums over n rows in fp32: 32 products to an instruction, then n / 32 of
    them and the joins (n / 32 + 96 roundings).  The output's rounding is half a step of bf16, 2^-8."""
    want, want_lse, mass, size = plain
    if not np.isfinite(want_lse):
        return np.isnan(o).all() and np.isnan(lse) if np.isnan(want_lse) else not o.any() and lse == want_lse
    dx = 2.0 ** -16 * size + 2.0 ** -22 * (abs(want_lse) + size + 32)
    steps = (n / 32 + 96) * 2.0 ** -24
    far = mass * (2.0 ** -16 + 2 * dx + 2 * steps) + 1e-37
    far = far + 2.0 ** -8 * (np.abs(want) + far)
    nan = np.isnan(want)
    return (np.isnan(o) == nan).all() and (np.abs(o - want)[~nan] <= far[~nan]).all() and \
        abs(lse - want_lse) <= dx + steps + 2.0 ** -22 * (1 + abs(want_lse))
