"""Inputs of the 8-bit attention whose results show by themselves how many bits of its operands were kept.

Scores: fp32 queries h + m + t of three bf16 parts, t at least 0.8 * 2^-18 under h < 1.25, all positive, against 4 codes that are not zero,
all positive: without t every score is 0.8 * 2^-18 / 1.25 = 41 * 2^-24 of itself too small.  With it, 4 codes times 3 parts are 12
additions, each off by at most 2^-23 of the sum so far (2^-24 rounded to nearest, twice that if a matrix instruction cuts off), the scales are
powers of two: 24 * 2^-24.

Weights: a query (1, 1024, 0 ..), so that scores are codes times a power of two, exactly.  Of a shard two entries count (the others' scores lie
hundreds below): one with the largest score, zero, whose value row is zero, and one whose weight p = exp(s - M) in [0.5, 1) keeps at least 0.7 * 2^-18 where bf16 takes two parts of it.  y = p V / (1 + p)
is then 0.7 * 2^-18 / p >= 44 * 2^-24 of itself off without the third part.  With it: p itself 4 * 2^-24 (argument times log2 e, |s - M| < 0.7: 1.5;
exponential: 2), also in the sum; product 3 additions of 2^-23; sums, factors and the quotient of the merge 8 * 2^-24: at most 22 * 2^-24."""
import numpy as np

import quant_reference as ref

SCORE_BAR, SCORE_SHORT = 26 * 2.0 ** -24, 41 * 2.0 ** -24
Y_BAR, Y_SHORT = 24 * 2.0 ** -24, 44 * 2.0 ** -24


def parts(x, n):
    """fp32 values as sums of n bf16 values, each the rounding of what the ones before left."""
    rest, out = np.asarray(x, np.float64), np.zeros(np.shape(x))
    for _ in range(n):
        part = ref.bf16(np.float32(rest)).astype(np.float64)
        out, rest = out + part, rest - part
    return out


def queries(rng, shape):
    h = 1 + rng.integers(0, 32, shape) / 128.0
    m = rng.integers(128, 256, shape) * 2.0 ** -17                       # below half a step of h, bf16 by itself
    t = rng.integers(26, 32, shape) * 2.0 ** -23                         # below half a step of m
    q = h + m + t
    assert (q == q.astype(np.float32)).all() and (q - parts(q, 2) >= 0.8 * 2.0 ** -18).all() and (parts(q, 3) == q).all()
    return q


def sparse_codes(rng, shape, fmt):
    """Positive codes in 4 places of a row, the largest among them, so that the scale is that of the format."""
    S, D = shape[-2:]
    rows = np.zeros((int(np.prod(shape[:-1])), D))
    at = rng.permuted(np.tile(np.arange(D), (len(rows), 1)), axis=1)[:, :4]
    values = rng.integers(1, 128, at.shape) if fmt == 0 else ref.E4M3[rng.integers(40, 127, at.shape)]
    np.put_along_axis(rows, at, values.astype(np.float64), 1)
    return rows.reshape(shape)


KEY_STEP = {0: 2.0 ** -7, 1: 2.0 ** -9}                                  # of the scores of a code


def weight_codes(fmt):
    """Codes v whose weight p = exp(-v KEY_STEP) keeps much where two parts are taken of it."""
    v = np.arange(1, 128.0) if fmt == 0 else ref.E4M3[8:127]
    p = np.exp(-v * KEY_STEP[fmt])
    good = v[(p >= 0.5) & (np.abs(p - parts(np.float32(p), 2)) >= 0.7 * 2.0 ** -18)]
    assert len(good) >= 5
    return good
