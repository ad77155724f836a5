"""Plain forms of the block-scaled FP8 KV cache in 64 bits, from the definitions,
on the host: what the kernels' results are compared with."""
import numpy as np

BLOCK = 64
# value of each E4M3 code (sign, 4 exponent bits of bias 7, 3 mantissa bits; S.1111.111 is NaN)
CODES = np.array([(-1.0 if c >> 7 else 1.0) * (np.nan if c & 127 == 127 else
                  (1 + (c & 7) / 8) * 2.0 ** ((c >> 3 & 15) - 7) if c >> 3 & 15 else (c & 7) / 8 * 2.0 ** -6)
                  for c in range(256)])


def exponent(amax):
    """The smallest e in [-100, 119] with amax <= 448 2^e."""
    e = -100
    while e < 119 and amax > 448.0 * 2.0 ** e:
        e += 1
    return e


def nearest(y):
    """Nearest E4M3 values (ties to even), saturated; NaN stays."""
    a = np.abs(y)
    with np.errstate(divide="ignore", invalid="ignore"):
        gap = 2.0 ** (np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
        r = np.minimum(np.round(a / gap) * gap, 448.0)
    r = np.where(np.isinf(y), 448.0, r)
    return np.where(np.isnan(y), np.nan, np.copysign(r, y))


def block_values(x):
    """(values of the codes, e, lowest, highest) of one block's rows x [rows, d] of a KV head."""
    x = np.asarray(x, np.float64)
    finite = np.abs(x[np.isfinite(x)])
    e = exponent(finite.max() if finite.size else 0.0)
    with np.errstate(invalid="ignore"):
        v = nearest(x / 2.0 ** e)
    return v, e, v.min(0), v.max(0)  # (min and max hand a NaN on)


def cache(x):
    """Values [n, h, d], scales [nb, h] and bounds [nb, 2, h, d] of rows x [n, h, d] (bounds in code units)."""
    n, h, d = x.shape
    nb = -(-n // BLOCK)
    v, s, b = np.zeros((n, h, d)), np.zeros((nb, h)), np.zeros((nb, 2, h, d))
    for i in range(nb):
        for j in range(h):
            r = slice(i * BLOCK, min(n, (i + 1) * BLOCK))
            v[r, j], e, b[i, 0, j], b[i, 1, j] = block_values(x[r, j])
            s[i, j] = 2.0 ** e
    return v, s, b


def attend(q, k, v, scale, pos, listed=None):
    """One query row over rows [0, pos] of k, v [n, d] (or the rows of the listed blocks, each as often as it is
    listed): (o, lse, sum of weight times |v|, sum of |v| times the largest weight of its block, sum of the products'
    magnitudes of a score)."""
    rows = np.arange(pos + 1)
    if listed is not None:
        rows = [np.arange(b * BLOCK, min(pos + 1, (b + 1) * BLOCK)) for b in listed if 0 <= b <= pos // BLOCK]
        rows = np.concatenate(rows) if rows else np.zeros(0, np.int64)
    d = k.shape[1]
    if rows.size == 0:
        return np.zeros(d), -np.inf, np.zeros(d), np.zeros(d), 0.0
    k, v = k[rows], v[rows]
    with np.errstate(invalid="ignore", over="ignore"):
        x = scale * (k @ q)
        m = x.max()
        p = np.exp(x - m)
        z = p.sum()
        p = p / z
        top = np.array([p[rows // BLOCK == b].max() for b in range(pos // BLOCK + 1) if (rows // BLOCK == b).any()])
        of = np.unique(rows // BLOCK, return_inverse=True)[1]
        return p @ v, m + np.log(z), p @ np.abs(v), top[of] @ np.abs(v), np.abs(scale * k * q).sum(1).max()


def close(o, lse, plain, d, fp8):
    """Whether a row's results are as near as the arithmetic allows.

    Scores: sums of d products in fp32 (d 2^-24 of their magnitudes); exponents in fp32 (2^-22 of the scores).  A score's
    error dx changes a weight by the factor 1 +- 2 dx (weight and sum).  Weights are rounded to 8 bits (2^-8), the output
    to bf16 (2^-8).

    fp8: weights go into the FP8 instruction in units where the largest of a block is above 128, as hi + lo / 16.  lo's
    codes are 2^-9 apart at least, so a weight is off by 2^-9 / 16 / 2 = 2^-14 where that is more than 2^-8 of it, which
    is 2^-21 of the block's largest.  The instruction's sums lose 2^-12 of the sum of the products' magnitudes."""
    want, want_lse, mass, top, size = plain
    if not np.isfinite(want_lse):
        return np.isnan(o).all() and np.isnan(lse) if np.isnan(want_lse) else not o.any() and lse == want_lse
    dx = d * 2.0 ** -24 * size + 2.0 ** -22 * (abs(want_lse) + size)
    weight = 2.0 ** -8
    far = mass * (weight + 2 * dx) + 1e-37
    if fp8:
        far = far + mass * 2.0 ** -12 + top * 2.0 ** -21
    far = far + 2.0 ** -8 * (np.abs(want) + far)
    nan = np.isnan(want)
    return (np.isnan(o) == nan).all() and (np.abs(o - want)[~nan] <= far[~nan]).all() and \
        abs(lse - want_lse) <= dx + 2.0 ** -22 * (1 + abs(want_lse))


def select(q, bounds, scales, n_sel, first, last, pos):
    """Blocks of one token and KV head: q [g, d], bounds [nb, 2, d] and scales [nb] of K."""
    mine = pos // BLOCK
    with np.errstate(invalid="ignore"):
        score = np.array([max(np.maximum(row * bounds[b, 0], row * bounds[b, 1]).sum() for row in q) * scales[b]
                          if not np.isnan(bounds[b]).any() and not np.isnan(q).any() else np.inf for b in range(mine + 1)])
    must = [b for b in range(mine + 1) if b < first or b > mine - last]
    rest = sorted((b for b in range(mine + 1) if b not in must), key=lambda b: (-score[b], b))
    keep = sorted(must + rest[:n_sel - len(must)])
    return keep + [-1] * (n_sel - len(keep))
