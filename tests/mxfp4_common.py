"""The MXFP4 format in 64 bits, from its definition in include/spex_tree.h: searches over the numbers that exist, no bit arithmetic."""

import numpy as np

NUMBERS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])  # in the order of their codes
BOUNDS = {"k": (-126, 125), "v": (-23, 13)}


def exponents(amax, which):
    """E of blocks with these largest magnitudes."""
    amax = np.asarray(amax, np.float64)
    m, e = np.frexp(amax)  # amax = m 2^e, 0.5 <= m < 1
    lo, hi = BOUNDS[which]
    return np.where(amax > 0, np.clip(e - 3, lo, hi), lo).astype(np.int64)


def nearest(x, e):
    """The nearest number times 2^e (one e per element), ties to the even code."""
    y = np.minimum(np.abs(x) / np.exp2(e.astype(np.float64)), 8.0)  # beyond 6 all the same; distances of 1e30 would not tell 4 from 6
    d = np.abs(y[..., None] - NUMBERS)
    best = d.min(-1, keepdims=True)
    code = np.where(d == best, np.arange(8) % 2 * 8 + np.arange(8), 99).min(-1) % 8  # among equals the even code
    return np.sign(x) * NUMBERS[code] * np.exp2(e.astype(np.float64))


def quantised(x, which):
    """What the cache holds for x [.., D], float64."""
    x = np.asarray(x, np.float64)
    b = x.reshape(*x.shape[:-1], -1, 32)
    e = np.broadcast_to(exponents(np.abs(b).max(-1), which)[..., None], b.shape)
    return nearest(b, e).reshape(x.shape)


def assert_held(got, x, off, which, what=""):
    """got: what the cache holds for values that are x within +- off, in 64 bits: for the block's E of some largest magnitude within
    reach, every value lies between what x - off and x + off round to."""
    got, x, off = (np.asarray(a, np.float64).reshape(-1, 32) for a in (got, x, off))
    top = np.argmax(np.abs(x), -1)[:, None]
    reach = np.abs(off).max(-1)
    amax = np.take_along_axis(np.abs(x), top, -1)[:, 0]
    fits = np.zeros(len(x), bool)
    for a in (np.maximum(amax - reach, 0), amax, amax + reach):
        e = np.broadcast_to(exponents(a, which)[:, None], x.shape)
        fits |= ((nearest(x - off, e) <= got) & (got <= nearest(x + off, e))).all(-1)
    assert fits.all(), (what, int((~fits).sum()), np.flatnonzero(~fits)[:4])


def attention(q, k, v, see, scale):
    """Rows q [R, D] over k, v [T, D], see [R, T]: out, lse, (sum of weights times |v|, sum of the visible |v|), sum |q||k| of the worst
    visible token; all in 64 bits."""
    x = scale * (q @ k.T)
    x = np.where(see, x, -np.inf)
    top = x.max(-1, keepdims=True)
    w = np.exp(x - top)
    total = w.sum(-1, keepdims=True)
    w /= total
    size = np.where(see, scale * (np.abs(q) @ np.abs(k).T), 0).max(-1)
    return w @ v, (top + np.log(total))[:, 0], (w @ np.abs(v), see.astype(float) @ np.abs(v)), size


def score_error(dim, size):
    """How far a scaled score may be off: a sum of `dim` fp32 products in any order, their magnitudes adding up to `size`, and its scaling."""
    return (dim + 4) * 2.0 ** -24 * size


def row_error(dim, tokens, size, mean):
    """Of an output; relative to the weighted mean of |v|, every weight by twice the scores' error (its own and its share of the sum's), the
    exponent's rounding (at most 2^-24 of it, up to 2^8 in magnitude where weights matter), the exponential and the weight's two fp16
    pieces (2^-21 each with room), sums over the tokens in fp32 in any order, twice (numerator, denominator), and the join.  Besides, absolutely: the pieces of a
    weight end at steps of 2^-24 where the row's largest weight is 2^7 or more, so each weight is off by up to 2^-31 of the largest."""
    relative = 2 * score_error(dim, size) + 2.0 ** -15 + 4 * 2.0 ** -21 + 2 * (tokens + 16) * 2.0 ** -24
    return relative[:, None] * mean[0] + 2.0 ** -31 * mean[1]
