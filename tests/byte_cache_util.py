"""The 8-bit cache of keys and values in plain 64-bit numpy, for tests: what a cache holds after its tokens came, what the tokens
stand for, attention over them, and how far fp32 sums with 16-bit operands may be off."""

import math

import numpy as np

BLOCK = 64


def to_half(x):
    """A token's values as they are kept: halves, saturated, NaN stays."""
    x = np.asarray(x, dtype=np.float32)
    return np.where(np.isnan(x), x, np.clip(x, -65504, 65504)).astype(np.float16)


def seal(block):
    """Codes and scale of one block [64][dim] of halves."""
    x = block.astype(np.float64)
    scale = np.float32(np.max(np.abs(x)) / 127) if not np.isnan(x).any() else np.float32(np.nan)
    if not scale > 0:
        return np.zeros(x.shape, dtype=np.int8), scale
    return np.rint(x / np.float64(scale)).astype(np.int8), scale


def contents(tokens):
    """tokens float32 [n][head][dim], already of the type's values -> (codes [head][block][64][dim], scales [head][block],
    rest half [head][n % 64][dim], values [n][head][dim] in 64 bits)."""
    n, heads, dim = tokens.shape
    h = to_half(tokens)
    whole = n // BLOCK
    codes = np.zeros((heads, whole, BLOCK, dim), dtype=np.int8)
    scales = np.zeros((heads, whole), dtype=np.float32)
    values = h.astype(np.float64)
    for i in range(heads):
        for b in range(whole):
            codes[i, b], scales[i, b] = seal(h[b * BLOCK:(b + 1) * BLOCK, i])
            values[b * BLOCK:(b + 1) * BLOCK, i] = codes[i, b].astype(np.float64) * np.float64(scales[i, b])
    return codes, scales, h[whole * BLOCK:].transpose(1, 0, 2), values


def attend(q, k, v, sees, scale):
    """q [row][head][dim], k / v [token][kv head][dim], sees [row][token] -> (out, lse, per-element sum of p |v| / sum of p,
    per (row, head) largest sum of |q||k|, largest |score|, largest sum of |k| times the query's largest) in 64 bits."""
    rows, heads, dim = q.shape
    group = heads // k.shape[1]
    out, mag = np.zeros((rows, heads, dim)), np.zeros((rows, heads, dim))
    lse, dot, top = np.full((rows, heads), -np.inf), np.zeros((rows, heads)), np.zeros((rows, heads))
    flat = np.zeros((rows, heads))
    for r in range(rows):
        idx = np.flatnonzero(sees[r])
        if len(idx) == 0:
            continue
        for h in range(heads):
            kk, vv, qq = k[idx, h // group], v[idx, h // group], q[r, h]
            s = kk @ qq * scale
            m = s.max()
            p = np.exp(s - m)
            total = p.sum()
            out[r, h], mag[r, h] = p @ vv / total, p @ np.abs(vv) / total
            lse[r, h] = m + math.log(total)
            dot[r, h] = (np.abs(kk) @ np.abs(qq)).max() * abs(scale)
            top[r, h] = np.abs(s).max()
            flat[r, h] = np.abs(kk).sum(axis=1).max() * np.abs(qq).max() * abs(scale)
    return out, lse, mag, (dot, top, flat)


HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
SMALLEST = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}        # half of the type's smallest number


def tolerance(kind, out, mag, scores, dim, tokens, largest):
    """Largest error of (out, lse), from the roundings of the definition's steps.

    A score: queries are whole numbers of steps of the row's largest / 32512 (bf16) or at most its 2^-21 (fp32, half), half a step off;
    against the tail they are halves (11 bits hold a 16-bit query but for parts below 2^-24 of the row's largest) or pairs.
    Products with codes are exact; those with the tail's halves are added in fp32 in up to two passes, each addition off by
    2^-24 of what the magnitudes sum up to; three factors in fp32.  A probability: its score's error, the exponential (2^-22),
    and as an operand 2^-12 (bf16 queries) or 2^-22, but never nearer than half of the smallest half, 2^-25, where the row's
    largest is at least 2^11 (pairs: 2^7 for single halves) over 2 (the reference is rounded up), times 1/2 to 1 for the value scale
    over its power of two (2^-12 where scales differ that much): 2^-35 of it for pairs, 2^-31 for single halves, times the values'
    largest magnitude for each token (the largest probability alone makes the sum that divides).  The sums are of the
    probabilities as they enter the products.  Sums over the tokens in fp32: 2^-24 each at most.  Then the output's own
    rounding, by half of its smallest number at least."""
    dot, top, flat = scores
    step = 1 / 65024 if kind == "bf16" else 2.0 ** -22
    score = dot * ((2 * dim + 8) * 2.0 ** -24 + 2.0 ** -22) + flat * (step + 2.0 ** -24) + top * 2.0 ** -22
    prob = score + 2.0 ** -22 + (2.0 ** -12 if kind == "bf16" else 2.0 ** -22)
    rel = 2 * prob + 2 * (tokens + 64) * 2.0 ** -24
    lse = prob + (tokens + 64) * 2.0 ** -24
    rounded = np.maximum(np.abs(out) * HALF_STEP[kind], SMALLEST[kind])
    return mag * rel[..., None] * 1.01 + rounded + tokens * largest * 2.0 ** (-31 if kind == "bf16" else -35) + 1e-30, lse + (top + 16) * 2.0 ** -23
