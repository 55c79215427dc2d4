"""Scored attention over the 8-bit cache in 64 bits, from its definition (numpy; shares no code with the library), with how far a kernel may be from it."""
import numpy as np

from q8_util import HALF_STEP


def visible(keys, rows, causal=False, prefix=0, first=None, end=None, window=0):
    """[rows, keys]: which tokens each row sees."""
    j = np.arange(keys)[None]
    e = np.clip(keys - rows + 1 + np.arange(rows), 0, None) if causal else np.full(rows, keys)
    if end is not None:
        e = np.minimum(e, np.maximum(end, 0))
    f = np.zeros(rows, np.int64) if first is None else np.maximum(first, 0).astype(np.int64)
    if window > 0:
        f = np.maximum(f, e - window)
    return (j < prefix) | ((j >= f[:, None]) & (j < e[:, None]))


def scored(q, k, v, see, form, dtype, cap=0.0, slopes=None, row_pos=None, key_pos=None):
    """(out, its bound, weights of the tokens, their bound) of rows q [m, heads, dh] over k, v [n, heads, dh].

    The bounds are those of a kernel that rounds each weight and the output to the type, and keeps everything else in 32 bits.  A score: dh products and sums and a
    scaling, 2^-24 each of the sum of magnitudes.  Its cap: exp2, a sum and a reciprocal, each off by a unit in the last place at most (2^-23), times twice the cap, 2^-20 of the
    cap in all; caps above 128 take a series for small scores, so that 2^-18 of the score itself bounds it, too.  The bias: a difference, a conversion and a product, 2^-22 of
    it.  The change to units of ln 2 and back: 2^-22 of the score."""
    m, heads, dh = q.shape
    n = k.shape[0]
    alpha, u = 1.0 / np.sqrt(dh), HALF_STEP[dtype]
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    total, dtotal = np.zeros(n), np.zeros(n)
    count = np.maximum(see.sum(axis=1, keepdims=True), 1)
    for h in range(heads):
        with np.errstate(invalid="ignore", over="ignore"):
            s = alpha * (q[:, h] @ k[:, h].T)
            ds = (dh + 8) * 2.0 ** -24 * alpha * (np.abs(q[:, h]) @ np.abs(k[:, h]).T)
        if cap:
            s = cap * np.tanh(s / cap)
            ds = ds + (np.abs(s) * 2.0 ** -18 + cap * 2.0 ** -32 if cap > 128 else cap * 2.0 ** -20)
        if slopes is not None:
            b = float(slopes[h]) * np.abs(row_pos[:, None].astype(np.float64) - key_pos[None].astype(np.float64))
            s = s - b
            ds = ds + np.abs(b) * 2.0 ** -22
        ds = ds + np.abs(s) * 2.0 ** -22
        if form == "softmax":
            t = np.where(see, s, -np.inf)
            top = np.max(t, axis=1, keepdims=True, initial=-1e300)
            w = np.where(see, np.exp(t - top), 0.0)
            w = w / np.maximum(w.sum(axis=1, keepdims=True), 1e-300)
            # (of the row: what its sum is off by, each term by as much as its own score)
            worst = np.sum(np.where(see, w * ds, 0.0), axis=1, keepdims=True)
            dx = w * (2 * (ds + worst) + 2.0 ** -20)
            dw = dx + w * 2 * u       # its own rounding, and the mean of the others' in the denominator
        else:
            w = np.where(see, s / (1.0 + np.exp(np.minimum(-s, 700.0))), 0.0) / count
            dx = np.abs(w) * 2.0 ** -20 + np.where(see, 1.1 * ds, 0.0) / count      # |SiLU'| < 1.1
            dw = dx + np.abs(w) * u
        if dtype == "fp16":      # weights below 2^-14 are multiples of 2^-24 (softmax: against a largest weight of at least 2^-8, the slack of its reference)
            dw = dw + np.where(see, 2.0 ** -25, 0.0) * (1.0 if form == "softmax" else 1.0 / count)
        av = np.abs(v[:, h])
        out[:, h] = w @ v[:, h]
        sums = np.abs(w) @ av
        bound[:, h] = dw @ av + n * 2.0 ** -24 * sums + u * (np.abs(out[:, h]) + dw @ av) + 2.0 ** -25
        total += np.abs(w).sum(axis=0)
        dtotal += dx.sum(axis=0)
    # (a sum of m * heads terms in 32 bits; exp2 of less than -126 is 0)
    return out, bound, total, dtotal + (m * heads + 2) * 2.0 ** -24 * total + m * heads * 2.0 ** -120
