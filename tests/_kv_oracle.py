"""Plain 64-bit restatement of the quantised cache and its attention (numpy),
for the tests: the format of include/akashic_mem.h."""
import math

import numpy as np

FLT_MAX = float(np.finfo(np.float32).max)


def _significant(x, bits):
    """x >= 0 rounded to so many significant bits, half to even."""
    unit = np.ldexp(1.0, np.frexp(x)[1] - bits)
    return np.rint(x / unit) * unit


def stored(x, bits):
    """The values that the cache stands for after the rows x (float64 [..., D]) are
    written."""
    x = np.asarray(x, np.float64)
    x = np.clip(np.where(np.isnan(x), 0.0, x), -FLT_MAX, FLT_MAX)
    if not x.size:
        return x
    a = np.abs(x).max(-1, keepdims=True)
    if bits == 8:
        s = np.maximum(_significant(a / 127, 8), 2.0 ** -100)
        return np.clip(np.rint(x / s), -127, 127) * s
    t = np.where(a == 0, -100, np.clip(np.frexp(a / 7)[1] - 1, -100, 125))
    g = x.reshape(*x.shape[:-1], -1, 16)
    r = np.abs(g).max(-1) / 7 / np.ldexp(1.0, t)
    e = np.clip(_significant(r, 5), 2.0 ** -15, 1.9375)
    s = (e * np.ldexp(1.0, t))[..., None]
    return (np.clip(np.rint(g / s), -7, 7) * s).reshape(x.shape)


def attend(q, keys, values, blocks, T, kv_len, q_start, *, causal=True, prefix=None, scale=None,
           cap=0.0, slopes=None, tags=None, q_tags=None, n_blocks=None):
    """q [n_q, Hq, D]; keys, values [slots, H, D] (stored values).  Returns out, lse, and
    for the tolerances: weight [n_q, Hq, D] = sum p |v|, top [n_q, Hq] = the largest |v|
    of the sequence's tokens, reach [n_q, Hq] = the largest |scale| sum_d |q_d k_d| of a seen key (small: sum |q| max |k| over the sequence's tokens), big [n_q, Hq] = sum over seen keys of
    max |v|, z [n_q, Hq] = the largest |z| with the bias' size."""
    n_q, hq, d = q.shape
    h = keys.shape[1]
    scale = scale or 1 / math.sqrt(d)
    out, lse = np.zeros((n_q, hq, d)), np.full((n_q, hq), -np.inf)
    weight, top = np.zeros((n_q, hq, d)), np.zeros((n_q, hq))
    reach, small, big, zmax = (np.zeros((n_q, hq)) for _ in range(4))
    for s in range(len(kv_len)):
        n, r0, r1 = int(kv_len[s]), int(q_start[s]), int(q_start[s + 1])
        tok = np.array([j for j in range(n) if blocks[s][j // T] >= 0], np.int64)
        at = np.array([blocks[s][j // T] * T + j % T for j in tok], np.int64)
        real = at if tags is None else at[tags[at] >= 0]
        if r1 == r0:
            continue
        pos = n - (r1 - r0) + np.arange(r1 - r0)
        seen = np.ones((r1 - r0, len(tok)), bool)
        if causal:
            first = int(prefix[s]) if prefix is not None else 0
            seen &= (tok[None] <= pos[:, None]) | (tok[None] < first)
        if tags is not None:
            seen &= (tags[at][None] == q_tags[r0:r1, None]) & (tags[at] >= 0)[None]
        some = seen.any(1)
        if not some.any():
            continue
        away = np.abs(pos[:, None] - tok[None])
        for hd in range(hq):
            K, V = keys[at, hd * h // hq], values[at, hd * h // hq]
            x = q[r0:r1, hd]
            z = scale * (x @ K.T)
            if cap:
                z = cap * np.tanh(z / cap)
            size = np.abs(z) + cap
            if slopes is not None:
                z = z - slopes[hd] * away
                size = np.abs(z) + cap + slopes[hd] * away
            z = np.where(seen, z, -np.inf)
            m = np.where(some, z.max(1, initial=-np.inf), 0.0)
            p = np.exp(z - m[:, None])
            total = np.where(some, p.sum(1), 1.0)
            rows = slice(r0, r1)
            lse[rows, hd] = np.where(some, m + np.log(total), -np.inf)
            p /= total[:, None]
            out[rows, hd] = p @ V
            weight[rows, hd] = p @ np.abs(V)
            top[rows, hd] = np.abs(values[real, hd * h // hq]).max(initial=0)
            big[rows, hd] = seen @ np.abs(V).max(1, initial=0)
            zmax[rows, hd] = np.where(seen, size, 0).max(1)
            reach[rows, hd] = abs(scale) * np.where(seen, np.abs(x) @ np.abs(K).T, 0).max(1)
            small[rows, hd] = abs(scale) * np.abs(x).sum(1) * np.abs(keys[real, hd * h // hq]).max(initial=0)
    return dict(out=out, lse=lse, weight=weight, top=top, reach=reach, small=small, big=big,
                z=zmax)


def tolerances(r, d, eps_half, bits):
    """Bounds of the error of out and lse, from the kernels' roundings.

    Scores: fp32 sums of d exact products and a few factors, (d + 8) 2^-24 of the
    sum of their sizes; a 4-bit key value v is held as v 2^-9 / 2^T in fp16, where the row's
    largest is at least 7 2^T, by two roundings of at most 2^-25: 2^-17 of the row's
    largest (of the tile's, where T is a tile's); a bf16 query value below 2^-14 of its row's to 2^-25 of
    it; cap, bias and the exponential's argument 2^-21 of their sizes.  A score off by t
    makes a weight off by t relative (both in the sum and in the total).  Weights: fp16,
    2^-11, with 2^-30 of the largest as the smallest step; the exponential 2^-21.
    Values: 4 bits, in the same way but as v 2^-10: 2^-16 of the sequence's largest.  The result is rounded once
    (eps_half of it; fp16 below 2^-14 has steps of 2^-24, so at least 2^-25)."""
    t = (d + 8) * 2.0 ** -24 * r["reach"] + 2.0 ** -21 * (r["z"] + 1)
    if bits == 4:
        t = t + 2.0 ** -17 * r["small"]
    rel = (2 * t + 2.0 ** -11 + 2.0 ** -20)[..., None]
    out = rel * r["weight"] + (2.0 ** -30 * r["big"])[..., None] + eps_half * np.abs(r["out"])
    if bits == 4:
        out = out + (2.0 ** -16 * r["top"])[..., None]
    lse = t + 2.0 ** -20 + 2.0 ** -22 * np.abs(np.where(np.isfinite(r["lse"]), r["lse"], 0))
    return out + (2.0 ** -25 if eps_half == 2.0 ** -11 else 1e-30), lse
