"""fp64 restatement of the 8-bit cache of uncompressed layers: codes, scales, and attention over them (numpy).

A cached number is code x scale; a scale belongs to a block of 16 tokens of one sequence and one KV head, keys and values
apart.  Writing new tokens sets the scale of every block that they reach to the smallest power of two 2^e, -100 <= e <= 100,
with which no new number exceeds the largest code, or leaves it where the block holds earlier tokens under a larger one;
the codes of these are re-expressed where it grows.  Codes are rounded to nearest, ties to even."""
from __future__ import annotations

import numpy as np

BLOCK = 16
LARGEST = {"int8": 127.0, "e4m3": 448.0}


def round_code(v, kind):
    v = np.asarray(v, dtype=np.float64)
    top = LARGEST[kind]
    if kind == "int8":
        return np.clip(np.rint(v), -top, top)
    # a number in [2^e, 2^(e+1)) has steps of 2^(e-3); below 2^-6 the step stays 2^-9
    _, ex = np.frexp(np.maximum(np.abs(v), 2.0 ** -6))
    step = np.ldexp(1.0, ex - 1 - 3)
    return np.clip(np.rint(v / step) * step, -top, top)


def scale_for(most, kind):
    """Smallest 2^e with most <= largest 2^e."""
    most = np.asarray(most, dtype=np.float64)
    e = np.full(most.shape, -100)
    live = most > 0
    e[live] = np.ceil(np.log2(most[live] / LARGEST[kind])).astype(int)
    e = np.where(live & (most > LARGEST[kind] * np.ldexp(1.0, e)), e + 1, e)      # (a logarithm may be off by an ulp)
    e = np.where(live & (most <= LARGEST[kind] * np.ldexp(1.0, e - 1)), e - 1, e)
    return np.ldexp(1.0, np.clip(e, -100, 100))


def write(codes, scales, new, length, kind):
    """codes [rows, H, d], scales [rows / 16, H] of one sequence (float64, changed in place); new [T, H, d] at positions
    length - T .. length - 1."""
    T = new.shape[0]
    for b0 in range((length - T) // BLOCK * BLOCK, length, BLOCK):
        start, end = max(b0, length - T), min(b0 + BLOCK, length)
        fresh = new[start - (length - T):end - (length - T)]
        s = scale_for(np.abs(fresh).max(axis=(0, 2)), kind)
        if start > b0:
            s = np.maximum(s, scales[b0 // BLOCK])
            codes[b0:start] = round_code(codes[b0:start] * (scales[b0 // BLOCK] / s)[None, :, None], kind)
        codes[start:end] = round_code(fresh / s[None, :, None], kind)
        scales[b0 // BLOCK] = s


def attention(k, v, q, group):
    """k, v [N, H, d] (numbers), q [H * group, d] rotated -> out [H * group, d] and, per head, the sum of |q_i k_i| / sqrt(d)
    at its largest (what score errors are relative to)."""
    n, _, d = k.shape
    out, size = np.zeros(q.shape), np.zeros(q.shape[0])
    for h in range(q.shape[0]):
        kk, vv = k[:, h // group], v[:, h // group]
        s = kk @ q[h] / np.sqrt(d)
        size[h] = (np.abs(kk) @ np.abs(q[h])).max() / np.sqrt(d)
        p = np.exp(s - s.max())
        out[h] = p @ vv / p.sum()
    return out, size
