"""Plain 64-bit restatement of the quantised cache and its attention (numpy),
for the tests: the format of include/akashic_mem.h, one row at a time."""
import math

import numpy as np

FLT_MAX = float(np.finfo(np.float32).max)


def _rne(x):
    return np.rint(x)                      # half to even


def stored_row(x, bits):
    """The values that the cache stands for after the row x (float64 [D]) is written."""
    x = np.clip(np.where(np.isnan(x), 0.0, x), -FLT_MAX, FLT_MAX)
    a = np.abs(x).max()
    if bits == 8:
        q = a / 127
        if q < 2.0 ** -100:
            s = 2.0 ** -100
        else:
            e = math.frexp(q)[1] - 8       # 8 significant bits
            s = math.ldexp(float(_rne(math.ldexp(q, -e))), e)
        return np.clip(_rne(x / s), -127, 127) * s
    t = -100 if a == 0 else min(125, max(-100, math.frexp(a / 7)[1] - 1))
    out = np.empty_like(x)
    for g in range(0, len(x), 16):
        r = np.abs(x[g:g + 16]).max() / 7 / 2.0 ** t
        if r <= 2.0 ** -15:
            e = 2.0 ** -15
        else:
            u = math.frexp(r)[1] - 5       # 5 significant bits
            e = min(1.9375, math.ldexp(float(_rne(math.ldexp(r, -u))), u))
        s = e * 2.0 ** t
        out[g:g + 16] = np.clip(_rne(x[g:g + 16] / s), -7, 7) * s
    return out


def stored(x, bits):
    x = np.asarray(x, np.float64)
    flat = x.reshape(-1, x.shape[-1])
    return np.stack([stored_row(r, bits) for r in flat]).reshape(x.shape) if len(flat) else x


def attend(q, keys, values, blocks, T, kv_len, q_start, *, causal=True, prefix=None, scale=None,
           cap=0.0, slopes=None, tags=None, q_tags=None, n_blocks=None):
    """q [n_q, Hq, D]; keys, values [slots, H, D] (stored values).  Returns out, lse, and
    for the tolerances: weight [n_q, Hq, D] = sum p |v|, top [n_q, Hq] = the largest |v|
    of the sequence's tokens, reach [n_q, Hq] = the largest |scale| sum_d |q_d k_d| of a seen key (small: sum |q| max |k|), big [n_q, Hq] = sum over seen keys of
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
        for i in range(r0, r1):
            pos = n - (r1 - r0) + (i - r0)
            seen = np.ones(len(tok), bool)
            if causal:
                seen &= (tok <= pos) | (tok < (int(prefix[s]) if prefix is not None else 0))
            if tags is not None:
                seen &= (tags[at] == q_tags[i]) & (tags[at] >= 0)
            if not seen.any():
                continue
            for hd in range(hq):
                K, V = keys[at[seen], hd * h // hq], values[at[seen], hd * h // hq]
                x = q[i, hd]
                z = scale * (K @ x)
                if cap:
                    z = cap * np.tanh(z / cap)
                away = np.abs(pos - tok[seen])
                if slopes is not None:
                    z = z - slopes[hd] * away
                    zmax[i, hd] = (slopes[hd] * away).max()
                zmax[i, hd] += np.abs(z).max() + cap
                m = z.max()
                p = np.exp(z - m)
                lse[i, hd] = m + math.log(p.sum())
                p /= p.sum()
                out[i, hd] = p @ V
                weight[i, hd] = p @ np.abs(V)
                top[i, hd] = np.abs(values[real, hd * h // hq]).max()
                big[i, hd] = np.abs(V).max(1).sum()
                reach[i, hd] = abs(scale) * (np.abs(K) @ np.abs(x)).max()
                small[i, hd] = abs(scale) * np.abs(x).sum() * np.abs(K).max()
    return dict(out=out, lse=lse, weight=weight, top=top, reach=reach, small=small, big=big,
                z=zmax)


def tolerances(r, d, eps_half, bits):
    """Bounds of the error of out and lse, from the kernels' roundings.

    Scores: fp32 sums of d exact products and a few factors, (d + 8) 2^-24 of the
    sum of their sizes; a 4-bit key value v is held as v 2^-9 / 2^T in fp16, where the row's
    largest is at least 7 2^T, by two roundings of at most 2^-25: 2^-17 of the row's
    largest; a bf16 query value below 2^-14 of its row's to 2^-25 of
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
