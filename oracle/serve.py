"""CPU oracle of rotary positions, the paged cache and the attention over it -- TEST INFRASTRUCTURE ONLY.

Straight from the definitions in include/hstu_attn.h, in float64 with numpy, one sequence and one head at a time; shares no
code with the GPU library.  `attention` also returns what its rounding errors are bounded by (see `attention_tolerance`).
"""
from __future__ import annotations

import numpy as np

U32 = 2.0 ** -24    # half a step of fp32, relative; bf16: 2 ** -8
UB16 = 2.0 ** -8


def rotate(x, positions, freq, interleaved=False, scale=1.0, backward=False):
    """x [rows, heads, d] turned by positions * freq (freq None: a copy)."""
    y = np.array(x, dtype=np.float64)
    if freq is None:
        return y
    half = len(freq)
    sign = -1.0 if backward else 1.0
    for j in range(half):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        # (the angle less whole turns in extended precision: numpy's cos of a large float64 is exact to its argument)
        angle = np.asarray(positions, dtype=np.float64) * float(freq[j])
        c, s = scale * np.cos(angle)[:, None], sign * scale * np.sin(angle)[:, None]
        xa, xb = np.asarray(x[:, :, a], dtype=np.float64), np.asarray(x[:, :, b], dtype=np.float64)
        y[:, :, a] = xa * c - xb * s
        y[:, :, b] = xb * c + xa * s
    return y


def rotation_tolerance(x, y, rotary, interleaved, scale, bf16, angle_error=0.0):
    """Per element.  c and s are off by 2 units (polynomial and rounding) and angle_error, two products and a sum round once
    each: (|x_a| + |x_b|) scale (4 u + angle_error); then one rounding to the output's type.  Copied elements are exact."""
    tol = np.zeros_like(y)
    half = rotary // 2
    ax = np.abs(np.asarray(x, dtype=np.float64))
    for j in range(half):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        tol[:, :, a] = tol[:, :, b] = (ax[:, :, a] + ax[:, :, b]) * abs(scale) * (4 * U32 + angle_error)
    if bf16:
        tol[:, :, :rotary] += UB16 * (np.abs(y[:, :, :rotary]) + tol[:, :, :rotary])
    return tol


def positions(off, rows, lens=None):
    """(sequence, position) of every row, sequence -1 for rows outside: the place in the sequence, or with lens the place in
    the cache."""
    seq, pos = np.full(rows, -1, dtype=np.int64), np.zeros(rows, dtype=np.int64)
    for b in range(len(off) - 1):
        s, e = int(off[b]), min(int(off[b + 1]), rows)
        for r in range(s, e):
            seq[r] = b
            pos[r] = r - s if lens is None else int(lens[b]) - (int(off[b + 1]) - s) + (r - s)
    return seq, pos


def place(table, num_pages, page_size, b, p):
    """(page, slot) of row p of sequence b, or None where there is none."""
    if p < 0 or p // page_size >= table.shape[1]:
        return None
    page = int(table[b, p // page_size])
    return (page, p % page_size) if 0 <= page < num_pages else None


def bucket(delta, nb, f):
    if delta <= 1:
        return 0
    e = int(delta).bit_length() - 1
    m = ((int(delta) << f) >> e) - (1 << f)
    return min(nb - 1, (e << f) + m)


def attention(q, k_pages, v_pages, table, lens, off, max_len, alpha, causal, ts=None, ts_pages=None, weights=None, f=0):
    """(o, sums): o [rows, heads, d_v], rows outside every sequence NaN.  sums: per element the three sums of
    attention_tolerance."""
    rows, heads, _ = q.shape
    pages, kv_heads, ps, dv = v_pages.shape
    group = heads // kv_heads
    o = np.full((rows, heads, dv), np.nan)
    sums = np.zeros((3, rows, heads, dv))
    most = table.shape[1] * ps
    for b in range(len(off) - 1):
        n = min(max(int(lens[b]), 0), most)
        m = int(off[b + 1]) - int(off[b])
        at = [place(table, pages, ps, b, p) for p in range(n)]
        there = np.array([a is not None for a in at], dtype=bool)
        pg = np.array([a[0] if a else 0 for a in at], dtype=np.int64)
        sl = np.array([a[1] if a else 0 for a in at], dtype=np.int64)
        for i in range(m):
            r = int(off[b]) + i
            seen = there & (np.arange(n) <= n - m + i) if causal else there
            o[r] = 0.0
            if not seen.any():
                continue
            w = 0.0
            if weights is not None:
                w = np.array([weights[bucket(abs(int(ts[r]) - int(ts_pages[g, s])), len(weights), f)]
                              for g, s in zip(pg[seen], sl[seen])], dtype=np.float64)
            for h in range(heads):
                k = np.asarray(k_pages[pg[seen], h // group, sl[seen]], dtype=np.float64)
                v = np.asarray(v_pages[pg[seen], h // group, sl[seen]], dtype=np.float64)
                qr = np.asarray(q[r, h], dtype=np.float64)
                x = alpha * (k @ qr + w)
                p = x / (1.0 + np.exp(-x))
                o[r, h] = p @ v / max_len
                av = np.abs(v) / max_len
                sums[0, r, h] = np.abs(p) @ av
                sums[1, r, h] = ((np.abs(x) + 8.0) * np.abs(p)) @ av
                sums[2, r, h] = abs(alpha) * (np.abs(k) @ np.abs(qr) + np.abs(w)) @ av
    return o, sums


def attention_tolerance(o, sums, d_qk, keys, bf16, out_bf16, one_term):
    """Per element, to first order.  A score is a sum of d_qk products (and the bias) in fp32: off by (d_qk + 1) u sum|q||k|, and
    SiLU's slope is below 1.1; its exponential's argument, exponential, sum and reciprocal round: (|x| + 8) u of P.  P enters the
    second product in fp32 (fp32), as two bf16 terms (2^-16) or one (2^-8).  The sum over keys rounds once a key.  Scaling and the
    output's rounding come last."""
    tol = U32 * (1.1 * (d_qk + 1) * sums[2] + sums[1] + (keys + 2) * sums[0])
    if bf16:
        tol = tol + (UB16 if one_term else UB16 * UB16) * sums[0]
    if out_bf16:
        tol = tol + UB16 * (np.abs(o) + tol)
    return tol + 1e-30
