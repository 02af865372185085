"""CPU oracle of the attention over a paged key-value cache (csrc/moe_kv.hip, csrc/moe_attn.hip) -- TEST
INFRASTRUCTURE ONLY, plain numpy in double.

    assign      block tables and slot maps of a step, request by request as include/moe.h defines them
    qk_norm_rope  per-head RMS norm and rotation of queries and keys, in doubles (nothing rounded), with the bound that the
                float32 arithmetic of a kernel has to keep
    attend      attention of one row over the tokens it sees, with such a bound
"""
from __future__ import annotations

import math

import numpy as np

U = 2.0 ** -24                                   # half a step of float32, relative


def assign(page_tokens, max_pages, pool_pages, T, cached, fresh, free_pages, free_head, block_table):
    """-> dict of the outputs of moe_kv_assign, the table after it, and the status bits."""
    table = np.array(block_table, dtype=np.int32, copy=True)
    B = len(cached)
    out = dict(seq_len=np.zeros(B, np.int32), row_start=np.zeros(B + 1, np.int32), positions=np.zeros(T, np.int32), slots=np.full(T, -1, np.int32),
               request=np.full(T, -1, np.int32))
    status, row, wanted, used = 0, 0, 0, 0
    head_ok = 0 <= free_head <= len(free_pages)
    left = len(free_pages) - free_head if head_ok else 0
    status |= 0 if head_ok else 1
    for b in range(B):
        c, f = int(cached[b]), int(fresh[b])
        had, new = max(c, 0), max(f, 0)
        held, total = -(-had // page_tokens), -(-(had + new) // page_tokens)
        need = total - held
        served = False
        if c < 0 or f < 0:
            status |= 1
        elif row + new > T:
            status |= 4
        elif total > max_pages:
            status |= 2
        else:
            wanted += need
            served = need == 0 or wanted <= left
            if not served:
                status |= 2
            elif need:
                table[b, held:total] = free_pages[free_head + wanted - need:free_head + wanted]
                used = wanted
        out["seq_len"][b] = had + new if served else had
        for i in range(min(new, max(0, T - row))):
            p = had + i
            out["positions"][row + i], out["request"][row + i] = min(p, 2 ** 31 - 1), b
            if served:
                page = int(table[b, p // page_tokens])
                if 0 <= page < pool_pages:
                    out["slots"][row + i] = page * page_tokens + p % page_tokens
                else:
                    status |= 1
        row += new
        out["row_start"][b + 1] = min(row, T)
    return dict(out, free_head=np.array([free_head + used], np.int32), block_table=table, status=status)


def qk_norm_rope(x, gamma, eps, inv_freq, positions, pairs):
    """x [T, heads, D] (exact in double), gamma [D] or None.  -> (values, bound): bound[t, h, d] is what float32 arithmetic
    may be off by before the last rounding.  With u = 2^-24: the sum of squares by chains of 8 and a tree of 5 additions loses
    14 u, half of it after the root, with the divisions, the root and both products 14 u in all; the angle, a float fraction of a turn, is off
    by 2 pi 2^-26 < 2 u, sine and cosine by 2 u more; the two products and their sum 2 u: 20 u of |a| + |b|."""
    x = np.asarray(x, np.float64)
    if gamma is not None:
        x = x / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps) * np.asarray(gamma, np.float64)
    y, size = x.copy(), np.abs(x)
    n = len(inv_freq)
    if n:
        angle = np.asarray(positions, np.float64)[:, None, None] * np.asarray(inv_freq, np.float64)
        c, s = np.cos(angle), np.sin(angle)
        first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if pairs else (slice(0, n), slice(n, 2 * n))
        a, b = x[..., first], x[..., second]
        y[..., first], y[..., second] = a * c - b * s, b * c + a * s
        size[..., first] = size[..., second] = np.abs(a) + np.abs(b)
    return y, 20 * U * size


def attend(q, k, v, scale, split_p):
    """q [G, D], k and v [n, D] (exact in double).  -> (out [G, D], lse [G], bound [G, D], lse_bound [G]).  The bound: a score is a chain
    of D products and sums, off by (D + 2) u sum |q k| scale, and with the running maximum and the exponent's argument by 6 u (|s| + |max|);
    twice that is the relative error of a weight against the sum of all weights, each of them off by another 4 u, the sums by u per
    addition in a chain (at most n / 4 + 32), and with split_p by 2^-15 more, as weights that are held in 16 bits."""
    n, D = k.shape
    if n == 0:
        return np.zeros_like(q), np.full(len(q), -np.inf), np.zeros_like(q), np.zeros(len(q))
    s = (q @ k.T) * scale
    m = s.max(-1, keepdims=True)
    p = np.exp(s - m)
    total = p.sum(-1, keepdims=True)
    es = (U * ((D + 2) * (np.abs(q) @ np.abs(k).T) * abs(scale) + 6 * (np.abs(s) + np.abs(m)))).max(-1, keepdims=True)
    w = p / total
    rel = 2 * es + U * (8 + n / 4 + 32) + (2.0 ** -15 if split_p else 0.0)
    return w @ v, (m + np.log(total))[:, 0], rel * (w @ np.abs(v)) + 1e-37, (rel + 4 * U * (1 + np.abs(m)))[:, 0]


def softmax_scale(D):
    return 1.0 / math.sqrt(D)
