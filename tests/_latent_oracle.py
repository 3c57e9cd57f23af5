"""Plain restatement of the rotation and of the latent cache's attention (numpy, 64 bits), for the
tests: the formulas of include/akashic_mem.h, with bounds of the kernels' roundings."""
import numpy as np


def rotate(x, positions, cos, sin, interleaved):
    """x [n, heads, d] (float32 values): the first 2 * cos.shape[1] of a row turned, in float32,
    each product and the sum rounded."""
    x = np.array(x, np.float32)
    r = 2 * cos.shape[1]
    c, s = cos[positions][:, None].astype(np.float32), sin[positions][:, None].astype(np.float32)
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    y, z = a * c - b * s, b * c + a * s
    out = x.copy()
    if interleaved:
        out[..., 0:r:2], out[..., 1:r:2] = y, z
    else:
        out[..., :r // 2], out[..., r // 2:r] = y, z
    return out


def attend(q, rows, blocks, T, kv_len, q_start, scale, bf16, R, *, causal=True, prefix=None, tags=None,
           q_tags=None, w_k=None, w_v=None):
    """q [n_q, H, ...], rows [slots, R + P] (values as stored).  Returns out, lse, and the bounds of their
    errors, tol and tol_lse.

    The bounds.  u: half a step of the cache's type (bf16 2^-8, fp16 2^-11, and 2^-25 where fp16 is
    subnormal).  Scores: fp32 sums of n products, (n + 8) 2^-24 of the sum of their sizes; the exponential and its
    argument 2^-21 of the score's size and 1.  Expanded: a key's values are fp32 sums of R
    products, rounded: u of their size more.  A score off by t makes a weight off by t, relative, in the sum and
    in the total.  Weights are rounded to the type: u; fp16's are held times at least 2^7 of the largest, so
    2^-25 2^-7 of the largest at least.  Values (expanded): as keys.  The result is rounded once."""
    n_q, H, _ = q.shape
    u, tiny = (2.0 ** -8, 1e-38) if bf16 else (2.0 ** -11, 2.0 ** -25)
    wide = R if w_k is None else w_v.shape[1]
    out, tol = np.zeros((n_q, H, wide)), np.full((n_q, H, wide), 1e-30)
    lse, tol_lse = np.full((n_q, H), -np.inf), np.full((n_q, H), 1e-30)
    for s in range(len(kv_len)):
        n, r0, r1 = int(kv_len[s]), int(q_start[s]), int(q_start[s + 1])
        if r1 == r0:
            continue
        tok = np.array([j for j in range(n) if blocks[s][j // T] >= 0], np.int64)
        at = np.array([blocks[s][j // T] * T + j % T for j in tok], np.int64)
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
        X = rows[at]
        for h in range(H):
            K, V = X, X[:, :R]
            kerr = verr = 0.0
            if w_k is not None:
                c = X[:, :R]
                k, v = c @ w_k[h].T, c @ w_v[h].T
                ks, vs = np.abs(c) @ np.abs(w_k[h]).T, np.abs(c) @ np.abs(w_v[h]).T
                K, V = np.concatenate((k, X[:, R:]), 1), v
                kerr = np.concatenate((u * np.abs(k) + (R + 8) * 2.0 ** -24 * ks + tiny, 0 * X[:, R:]), 1)
                verr = u * np.abs(v) + (R + 8) * 2.0 ** -24 * vs + tiny
            x = q[r0:r1, h]
            z = scale * (x @ K.T)
            reach = abs(scale) * (np.abs(x) @ np.abs(K).T)
            t = (K.shape[1] + 8) * 2.0 ** -24 * reach + 2.0 ** -21 * (np.abs(z) + 1)
            if w_k is not None:
                t = t + abs(scale) * (np.abs(x) @ kerr.T)
            z = np.where(seen, z, -np.inf)
            t = np.where(seen, t, 0).max(1)
            m = np.where(some, z.max(1, initial=-np.inf), 0.0)
            p = np.exp(z - m[:, None])
            total = np.where(some, p.sum(1), 1.0)
            i = slice(r0, r1)
            lse[i, h] = np.where(some, m + np.log(total), -np.inf)
            p /= total[:, None]
            o = p @ V
            out[i, h] = o
            big = np.where(seen, 1.0, 0.0) @ np.abs(V) / total[:, None]
            weight = p @ np.abs(V)
            e = (2 * t + u + 2.0 ** -20)[:, None] * weight + u * np.abs(o) + tiny
            if not bf16:
                e = e + 2.0 ** -32 * big
            if w_k is not None:
                e = e + p @ verr
            tol[i, h] = np.where(some[:, None], e, 1e-30)
            tol_lse[i, h] = np.where(some, t + 2.0 ** -20 + 2.0 ** -22 * np.abs(np.where(some, lse[i, h], 0)), 1e-30)
    return dict(out=out, lse=lse, tol=tol, tol_lse=tol_lse)
