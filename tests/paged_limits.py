"""Attention of drafted trees over the paged cache in 64 bits, with a limit on the error of each (row, head) as a whole.

With weights p_t and values v_t, an error d_t of score t (which the sum of the weights shares) moves the output by p_t d_t (v_t - out),
an error e_t of the weight beside its value alone (it is rounded after the sum has taken it) by p_t e_t v_t.  The errors of different
tokens have no common direction, so their root mean square adds up to
    n = sqrt(sum_t p_t^2 (|v_t - out|^2 d_t^2 + |v_t|^2 e_t^2))
which falls with the number of tokens as the output itself does; four times that is the limit.  As root mean squares:
    d_t   bf16 calls round the rotated query to fp16: 2^-11 / sqrt(3) of every product's factor, sqrt(sum_d (q_d k_d)^2) in all.
          fp32 calls: 18 matrix instructions, each of which cuts up to 2^-23 off the running sum, half of it on average; the sums,
          of codes less 8, are taken as twice sqrt(sum_d (q_d k_d)^2).  Either way 2^-22 of the score for the fp32 steps after it and
          2^-22 for the exponential
    e_t   fp16: 2^-11 / sqrt(3); in two parts: 2^-22
To that comes the rounding of the result, 2^-8 of it for bf16 and 2^-23 for fp32, and for fp32, whose blocks are summed by six matrix
instructions over codes less 8 and zero-points less 8 (at most 8 each), 6 x 2^-23 of sum_t p_t 16 s_t in every dimension, s_t the
value's scale (a vector of zeros takes no part).
"""
import numpy as np

import paged_ref as ref

D = ref.D


def seen_by(mask, n, first, length):
    """[n, length] truth values: the positions that rows of a request see.  mask: int32 [n, words] or None."""
    j = np.arange(length)[None] - first
    if mask is None:
        return j <= np.arange(n)[:, None]
    bits = np.ascontiguousarray(mask).view(np.uint32)
    jj = np.clip(j[0], 0, 32 * bits.shape[1] - 1)
    return (j < 0) | ((j < 32 * bits.shape[1]) & ((bits[:, jj >> 5] >> (jj & 31).astype(np.uint32)) & 1 == 1))


def one_head(q, k, v, seen, scale, fp32, value_scale=None):
    """q [m, D] (rotated), k, v [T, D], seen [m, T], value_scale [T] -> out [m, D] in 64 bits and the limits [m]."""
    score = np.where(seen, q @ k.T * scale, -np.inf)
    spread = np.sqrt((q * q) @ (k * k).T) * scale
    top = score.max(axis=1, keepdims=True, initial=-1e300)
    p = np.exp(score - top)
    p /= np.maximum(p.sum(axis=1, keepdims=True), 1e-300)
    out = p @ v
    d = (9 * 2.0 ** -23 * 2 * spread if fp32 else 2.0 ** -11 / np.sqrt(3) * spread) + 2.0 ** -22 * (1 + np.where(seen, np.abs(score), 0))
    e = 2.0 ** -22 if fp32 else 2.0 ** -11 / np.sqrt(3)
    own = (v * v).sum(1)[None]
    apart = np.maximum(own - 2 * out @ v.T + (out * out).sum(1)[:, None], 0)           # |v_t - out|^2
    n = np.sqrt((p * p * (apart * d * d + own * e * e)).sum(axis=1))
    limit = 4 * n + (2.0 ** -23 if fp32 else 2.0 ** -8) * np.linalg.norm(out, axis=1) + 1e-36
    if fp32 and value_scale is not None:
        limit += 6 * 2.0 ** -23 * 16 * np.sqrt(D) * (p @ np.where(v.any(axis=1), value_scale, 0))
    return out, limit


def attention(q, pool, table, page_tokens, row_start, first, mask=None, q_had=0, scale=None, fp32=True):
    """-> out fp64 [total, Hq, D] and the limit of each row and head's error, [total, Hq].  Positions without a page are seen by nobody."""
    total, Hq, D = q.shape
    H = pool.shape[1]
    G = Hq // H
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    qr = ref.rotate(q, q_had)
    out, limit = np.zeros((total, Hq, D)), np.zeros((total, Hq))
    held = {}
    for r in range(len(first)):
        a, n, f = int(row_start[r]), int(row_start[r + 1] - row_start[r]), int(first[r])
        length = max(0, min(f + n, table.shape[1] * page_tokens))
        if n <= 0 or length == 0:
            continue
        key = (tuple(table[r]), length)                                               # requests may share their pages
        if key not in held:
            parts = ref.cached(pool, table, page_tokens, r, length)
            have = np.repeat([0 <= int(t) < pool.shape[0] for t in table[r]], page_tokens)[:length]
            held = {key: (ref.dequant(*parts[:3]), ref.dequant(*parts[3:]), have, np.where(have[:, None], parts[4], 0).astype(np.float64))}
        k, v, have, vs = held[key]
        seen = seen_by(None if mask is None else mask[a:a + n], n, f, length) & have
        for h in range(H):
            o, lim = one_head(qr[a:a + n, h * G:(h + 1) * G].reshape(n * G, D), np.where(have[:, None], k[:, h], 0), np.where(have[:, None], v[:, h], 0),
                              np.repeat(seen, G, 0), scale, fp32, vs[:, h])
            out[a:a + n, h * G:(h + 1) * G], limit[a:a + n, h * G:(h + 1) * G] = o.reshape(n, G, D), lim.reshape(n, G)
    return out, limit
