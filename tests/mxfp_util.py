"""Plain 64-bit forms of the operators on tables held in 4 bits and of draws (numpy, written from the definitions), shared by their tests."""
import math

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
MIDS = (LEVELS[1:] + LEVELS[:-1]) / 2


def blocks_of(dim):
    return (dim + 31) // 32


def quantise(x):
    """Codes [n, 16 blocks] and scale bytes [n, blocks] of rows in 64 bits."""
    x = np.asarray(x, dtype=np.float64)
    n, dim = x.shape
    nb = blocks_of(dim)
    v = np.zeros((n, nb * 32))
    v[:, :dim] = x
    v = v.reshape(n, nb, 32)
    finite = np.isfinite(v).all(2)
    v = np.where(finite[:, :, None], v, 0.0)
    largest = np.abs(v).max(2)
    e = np.where(largest > 0, np.maximum(np.frexp(largest)[1] - 3, -127), -127)
    a = np.abs(v) * np.exp2(-e.astype(np.float64))[:, :, None]
    code = np.searchsorted(MIDS, a, side="left")             # a value on the border to the next level is counted below it ..
    tie = (code < 7) & (a == MIDS[np.minimum(code, 6)])
    code = np.where(tie & (code % 2 == 1), code + 1, code)   # .. and goes to the even one
    code = (code + 8 * np.signbit(v)).astype(np.uint8)
    code[~finite] = 0
    code = code.reshape(n, nb * 16, 2)
    scales = np.where(finite, e + 127, 255).astype(np.uint8)
    return code[:, :, 0] | (code[:, :, 1] << 4), scales


def values(codes, scales, dim):
    """What codes and scale bytes stand for, in 64 bits."""
    codes, scales = np.asarray(codes), np.asarray(scales)
    c = np.stack((codes & 15, codes >> 4), axis=2).reshape(codes.shape[0], -1)
    unit = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    with np.errstate(invalid="ignore"):
        v = np.where(c >= 8, -1.0, 1.0) * LEVELS[c % 8] * np.repeat(unit, 32, axis=1)
    return v[:, :dim]


def score_bound(q, w, kind, scale, half_step, tiny=0.0):
    """Scores of q [T, d] and w [V, d] (64 bits) with the most that a score may be off: slices, fp32 sums, the result's rounding.

    Slices: the last digit of a block whose largest magnitude lies in [2^e, 2^(e + 1)) stands for 2^(e - 23) (fp32, five slices) or
    2^(e - 18) (four), so a value is off by at most half of that: 2^-24 or 2^-19 of the block's largest.  Sums: a step of 64 columns adds
    its products to a partial sum whose magnitude is at most A = sum |q w|; the result and the alignment of its terms cost at most
    2^-23 A each; slices but the first add 1/31 of that.  The product with the scale rounds once."""
    T, d = q.shape
    nb = blocks_of(d)
    pad = np.zeros((T, nb * 32))
    pad[:, :d] = np.abs(q)
    largest = np.repeat(pad.reshape(T, nb, 32).max(2), 32, axis=1)[:, :d]
    slice_error = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -19, "fp16": 2.0 ** -19, "mxfp4": 0.0}[kind]
    s = (q @ w.T) * scale
    size = (np.abs(q) @ np.abs(w).T) * scale
    steps = (d + 63) // 64
    bound = (largest * slice_error) @ np.abs(w).T * scale + size * (2 * steps + 2) * 2.0 ** -23 * (32 / 31)
    return s, bound + (np.abs(s) + bound) * (2.0 ** -24 + half_step) + tiny


FLT_MAX = float(np.finfo(np.float32).max)


def kept_rows(scores, allowed, temperature, top_k, top_p, min_p):
    """Ids of the kept rows ascending with their weights (extended precision); scores: 64-bit, allowed: bool or None."""
    s = np.minimum(np.asarray(scores, dtype=np.float64), FLT_MAX)
    counts = s > -np.inf                                      # neither NaN nor -infinity
    if allowed is not None:
        counts &= allowed
    ids = np.nonzero(counts)[0]
    if not len(ids):
        return ids, np.zeros(0, dtype=np.longdouble)
    if not temperature > 0:
        temperature, top_k = 1.0, 1
    ids = ids[np.lexsort((ids, -s[ids]))]
    z = (s[ids] - s[ids[0]]).astype(np.longdouble)
    z = np.zeros_like(z) if math.isinf(temperature) else z / np.longdouble(temperature)
    w = np.exp(z)
    if top_k > 0:
        ids, w = ids[:top_k], w[:top_k]
    keep = np.ones(len(ids), dtype=bool)
    if top_p < 1:
        before = np.concatenate(([np.longdouble(0)], np.cumsum(w)[:-1]))
        keep = before < np.longdouble(top_p) * w.sum()
        keep[0] = True
    if min_p > 0:
        keep &= w >= min(min_p, 1.0)
    ids, w = ids[keep], w[keep]
    order = np.argsort(ids)
    return ids[order], w[order]


def draws(scores, allowed, temperature, top_k, top_p, min_p, uniforms):
    """ids, log probabilities, number of kept rows."""
    ids, w = kept_rows(scores, allowed, temperature, top_k, top_p, min_p)
    if not len(ids):
        return np.full(len(uniforms), -1), np.full(len(uniforms), -np.inf), 0
    mass = np.cumsum(w)
    positive = np.nonzero(w > 0)[0][-1]
    u = np.asarray(uniforms, dtype=np.float64)
    u = np.where(u > 0, u, 0.0)                              # NaN as well
    at = np.minimum(np.searchsorted(mass, u.astype(np.longdouble) * mass[-1], side="right"), positive)
    return ids[at], np.log(w[at] / mass[-1]).astype(np.float64), len(ids)
