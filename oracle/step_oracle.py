"""Plain CPU oracle of what a step does around the paged key/value cache.  TEST INFRASTRUCTURE ONLY: it shares nothing with the library.

* advance        : the tables of a step, a sequence, an entry and a row at a time.
* rope64         : norm, rotation and matrix in fp64, with the error bound of an fp32 / fp16 computation.
* scored64       : attention in fp64 with capped scores, slopes and a prefix, with what its bound needs.
"""
from __future__ import annotations

import math

import numpy as np

D = 128


def advance(held, keep, rows, table, width, page, pages, ring, taken, given, T):
    """table: a list of rows (lists, at least `width` long), ring: a list; both are changed.  Returns (row_starts, lengths, (taken, given, missing),
    positions, slots)."""
    B = len(held)
    starts, lengths, want = [0], [], []
    for b in range(B):
        h = max(0, held[b])
        k = min(max(0, keep[b]), h)
        n = min(max(0, rows[b]), 2 ** 31 - 1 - k, T - starts[b])
        have, need = (min(-(-x // page), width) for x in (h, k + n))
        starts.append(starts[b] + n)
        lengths.append(k + n)
        want.append((have, need))
    count = sum(max(0, need - have) for have, need in want)
    free = min(max(given - taken, 0), len(ring))
    enough, got, back = count <= free, [], []
    for b, (have, need) in enumerate(want):
        for j in range(have, need):
            table[b][j] = ring[(taken + len(got)) % len(ring)] if enough else -1
            got.append(j)
        for j in range(need, have):
            if 0 <= table[b][j] < pages:
                back.append(table[b][j])
                if not enough:
                    table[b][j] = -1                                           # the call is made again: it finds no page there
    for i, p in enumerate(back):
        ring[(given + i) % len(ring)] = p
    positions, slots = [-1] * T, [-1] * T
    for b in range(B):
        n = starts[b + 1] - starts[b]
        for i in range(n):
            pos = lengths[b] - n + i
            positions[starts[b] + i] = pos
            if pos // page < width and 0 <= table[b][pos // page] < pages:
                slots[starts[b] + i] = table[b][pos // page] * page + pos % page
    return starts, lengths, (taken + (count if enough else 0), given + len(back), 0 if enough else count - free), positions, slots


def turned64(x, w, eps, positions, frequencies, interleaved):
    """fp64 rows [T, heads, 128] after norm and rotation, and (|a| + |b|) of every number's pair (itself where it is not turned)."""
    y = np.asarray(x, dtype=np.float64)
    if w is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * np.asarray(w, dtype=np.float64)
    out, size = y.copy(), np.abs(y)
    half = len(frequencies)
    for i, f in enumerate(frequencies):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = np.asarray(positions, dtype=np.float64)[:, None] * f
        c, s = np.cos(angle), np.sin(angle)
        out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
        size[..., a] = size[..., b] = np.abs(y[..., a]) + np.abs(y[..., b])
    return out, size


def turned_bound(size):
    """Before the rounding to fp16.  The norm's factor: nine additions behind each other, each 2^-24 of the sum, halved by the root, and 2^-23 of the root's
    instruction: 2^-21; cosine and sine: the terms left out 2^-25, four fmas and the angle 2^-22; the weight, two products and a sum 2^-22 in all.
    Less than 2^-20 of |a| + |b|."""
    return size * 2.0 ** -20


def half_bound(y, off):
    """Of a number that is off by `off` and then rounded to fp16."""
    return off + (np.abs(y) + off) * 2.0 ** -11 + 2.0 ** -25


def rope64(x, w, eps, positions, frequencies, interleaved, P=None):
    """(out, bound) fp64 [T, heads, 128]; P fp16 [heads or 1, 128, 128]."""
    y, size = turned64(x, w, eps, positions, frequencies, interleaved)
    off = half_bound(y, turned_bound(size))
    if P is None:
        return y, off
    out, bound = np.empty_like(y), np.empty_like(y)
    for h in range(y.shape[1]):
        M = np.asarray(P[h % len(P)], dtype=np.float64)
        out[:, h] = y[:, h] @ M
        # 128 products in eight instructions of 16: each sum is off by 2^-24 of the numbers' sizes an addition
        bound[:, h] = half_bound(out[:, h], off[:, h] @ np.abs(M) + 130 * 2.0 ** -24 * ((np.abs(y[:, h]) + off[:, h]) @ np.abs(M)))
    return out, bound


def scored64(q, k, v, seen, scale, positions, cap, slope, k_step, v_step, k_bits=4):
    """One head: q [n, 128], k, v [L, 128], seen [n, L], positions [n], the tokens' steps [L].  Returns out [n, 128] (zeros for a row that sees nothing) and for
    the bound A = sum_j w_j |v_j|, S = sum_j w_j v_step_j, and what errors of the scores do, E = sum_j w_j d_j (|v_j| + |out|).  The error d_j of a score:
    of the product as for plain scores (cache_oracle.attention64; tanh's slope is at most one); of the cap 2^-21 of it, where it is beyond 177 2^-19
    of the score; of the score and its distance's part, base 2, a product and a sum of each 2^-22."""
    q = np.asarray(q, dtype=np.float64)
    n, L = seen.shape
    out, A, S, E = np.zeros((n, D)), np.zeros((n, D)), np.zeros(n), np.zeros((n, D))
    for i in range(n):
        j = np.flatnonzero(seen[i])
        if len(j) == 0:
            continue
        s = scale * (k[j] @ q[i])
        a = np.abs(q[i])
        d = abs(scale) * k_step[j].max() * (280 * 2.0 ** -24 * (2 ** k_bits - 1) * a.sum() + 132 * 2.0 ** -18 * a.max()) + np.zeros(len(j))
        if cap:
            s = cap * np.tanh(s / cap)
            d = d + (cap * 2.0 ** -21 if cap < 177 else np.abs(s) * 2.0 ** -19 + 2.0 ** -22)
        low = slope * np.abs(positions[i] - j)
        d = d + (np.abs(s) + abs(low)) * 2.0 ** -22
        s = s - low
        w = np.exp(s - s.max())
        w /= w.sum()
        out[i] = w @ v[j]
        A[i], S[i] = w @ np.abs(v[j]), w @ v_step[j]
        E[i] = (w * d) @ np.abs(v[j]) + (w @ d) * np.abs(out[i])
    return out, A, S, E


def scored_bound(out, A, S, E, tokens, v_bits=4, capped=True):
    """As cache_oracle.attention_bound with what errors of the scores do (E, to first order: 2^-6 of it more).  Of many rows with a cap references are raised so that the largest
    product is 2^2 there and not 2^7, up to 2^14 tokens: a product in fp16's subnormals loses 2^-25 at most, 2^-27 of the largest, which is S at most in sum: 2^b - 1 units of a
    code each."""
    from oracle.cache_oracle import attention_bound
    lost = tokens * (2.0 ** -27 - 2.0 ** -32) if capped and tokens <= 2 ** 14 else 0.0
    return attention_bound(out, A, S, np.zeros(len(out)), tokens, v_bits) + E * (1 + 2.0 ** -6) + S[:, None] * ((2 ** v_bits - 1) * lost)


def slopes(heads):
    return np.array([2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)], dtype=np.float32)


def turns_exact(frequency):
    """Nearest multiple of 2^-64 of a turn, from a fraction's digits: pi to 60 digits."""
    from fractions import Fraction
    pi = Fraction("3.14159265358979323846264338327950288419716939937510582097494")
    x = Fraction(frequency) / (2 * pi)
    return int(math.floor(x * 2 ** 64 + Fraction(1, 2))) % 2 ** 64
