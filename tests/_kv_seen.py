"""Bounds of the attention's errors by what a row sees: the keys and values that its mask
leaves, each value with its weight.  (_kv_oracle.tolerances takes the largest of all
of the sequence's tokens, seen or not.)"""
import math

import numpy as np


def add(want, q, keys, values, blocks, T, kv_len, q_start, *, causal=True, prefix=None, scale=None,
        cap=0.0, slopes=None, tags=None, q_tags=None, **_):
    """What tolerances() needs, added to the result of _kv_oracle.attend for the same
    arguments, each [n_q, Hq]: own = |scale| sum |q| times the largest |k| of a seen key,
    low = |scale| max |q| times the largest sum |k| of one, wtop = sum over seen keys of p max |v|,
    peak = the largest p max |v|, most = the largest |v| seen, count = keys seen, near = the largest p
    times the sum of max |v| over seen values below 56."""
    n_q, hq, d = q.shape
    h = keys.shape[1]
    scale = scale or 1 / math.sqrt(d)
    own, low, wtop, peak, most, count, near = (np.zeros((n_q, hq)) for _ in range(7))
    for s in range(len(kv_len)):
        n, r0, r1 = int(kv_len[s]), int(q_start[s]), int(q_start[s + 1])
        tok = np.array([j for j in range(n) if blocks[s][j // T] >= 0], np.int64)
        if r1 == r0 or not len(tok):
            continue
        at = np.array([blocks[s][j // T] * T + j % T for j in tok], np.int64)
        pos = n - (r1 - r0) + np.arange(r1 - r0)
        seen = np.ones((r1 - r0, len(tok)), bool)
        if causal:
            first = int(prefix[s]) if prefix is not None else 0
            seen &= (tok[None] <= pos[:, None]) | (tok[None] < first)
        if tags is not None:
            seen &= (tags[at][None] == q_tags[r0:r1, None]) & (tags[at] >= 0)[None]
        away = np.abs(pos[:, None] - tok[None])
        rows = slice(r0, r1)
        for hd in range(hq):
            K, V = keys[at, hd * h // hq], values[at, hd * h // hq]
            x = q[rows, hd]
            z = scale * (x @ K.T)
            if cap:
                z = cap * np.tanh(z / cap)
            if slopes is not None:
                z = z - slopes[hd] * away
            lse = want["lse"][rows, hd][:, None]
            p = np.where(seen, np.exp(np.where(seen, z, 0) - np.where(np.isfinite(lse), lse, 0)), 0)
            ktop, vtop = np.abs(K).max(1), np.abs(V).max(1)
            own[rows, hd] = abs(scale) * np.abs(x).sum(1) * np.where(seen, ktop, 0).max(1)
            low[rows, hd] = abs(scale) * np.abs(x).max(1) * np.where(seen, np.abs(K).sum(1), 0).max(1)
            wtop[rows, hd] = p @ vtop
            peak[rows, hd] = (p * vtop).max(1)
            most[rows, hd] = np.where(seen, vtop, 0).max(1)
            count[rows, hd] = seen.sum(1)
            near[rows, hd] = p.max(1) * (seen @ np.where(vtop < 56, vtop, 0))
    want.update(own=own, low=low, wtop=wtop, peak=peak, most=most, count=count, near=near)
    return want


def tolerances(r, d, eps_half, bits, dtype):
    """Bounds of the error of out and lse, from the kernels' roundings.

    Scores: fp32 sums of d exact products and a few factors, (d + 8) 2^-24 of the sum of
    their sizes; cap, bias and the exponential's argument 2^-21 of their sizes.  A 4-bit
    key is held as v 2^-9 / 2^T in fp16, T its own row's exponent, by two roundings of at most
    2^-25: its largest is at least 7 2^T, so 2^-17 of it.  A bf16 query value below 2^-14 of
    its row's largest to 2^-25 of it.  A score off by t makes a weight off by t
    relative (in the sum and in the total).
    Weights: the exponential 2^-21; times the value's power of two, fp16: 2^-11, or 2^-25
    where the greatest of the row's so far was at least 2^2, so 2^-27 of it, times the
    value's 13.6 at most where the greatest's largest is 7 or more (8 bits: 127 and
    64): 2^-26 of the row's greatest p max |v| a key.  In the kernel for many rows 4-bit values
    within a window below 56 are as they are and their weights without a power of two: 2^-27 of the
    greatest weight, 2^-26 of it times max |v|.  Weights below 2^-126 are 0.
    Values: 4 bits, rounded as the keys: 2^-17 of their own row's largest, with its weight.
    The result is rounded once (fp16 below 2^-14 has steps of 2^-24)."""
    t = (d + 8) * 2.0 ** -24 * r["reach"] + 2.0 ** -21 * (r["z"] + 1)
    if bits == 4:
        t = t + 2.0 ** -17 * r["own"]
    if dtype == "bf16":
        t = t + 2.0 ** -25 * r["low"]
    rel = (2 * t + 2.0 ** -11 + 2.0 ** -20)[..., None]
    out = rel * r["weight"] + eps_half * np.abs(r["out"])
    out = out + (2.0 ** -26 * r["count"] * r["peak"] + 2.0 ** -126 * r["most"])[..., None]
    if bits == 4:
        out = out + (2.0 ** -17 * r["wtop"] + 2.0 ** -26 * r["near"])[..., None]
    lse = t + 2.0 ** -20 + 2.0 ** -22 * np.abs(np.where(np.isfinite(r["lse"]), r["lse"], 0))
    return out + (2.0 ** -25 if dtype == "fp16" else 1e-30), lse
