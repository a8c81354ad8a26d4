"""Plain CPU oracle of the paged key/value cache and its attention.  TEST INFRASTRUCTURE ONLY: it shares nothing with the library.

* grid32           : asymmetric b-bit groups (Sec. 4.1 "Quantization") by the sequence of correctly rounded fp32 operations that the
                     write without a matrix is defined by; numpy's float32 arithmetic is IEEE.
* pack / unpack    : code k of a group at bits [b k, b k + b) of its bytes read as one little-endian integer, bit by bit.
* Pages            : pages, page table and lengths of a batch on the host, with the write and the read by loops over tokens.
* attention64      : softmax attention in fp64 over the de-quantized values, one (sequence, head) at a time, with what the error
                     bound of an fp32 / fp16 computation needs.
"""
from __future__ import annotations

import numpy as np

D = 128


def grid32(y, clip, bits):
    """y fp16 [..., 128] -> (codes uint8 [..., 128], steps fp16 [...], zero points uint8 [...])."""
    f = np.float32
    y = np.asarray(y, dtype=np.float16).astype(f)
    top = f(2 ** bits - 1)
    mx = f(clip) * np.maximum(y.max(-1), f(0))
    mn = f(clip) * np.minimum(y.min(-1), f(0))
    with np.errstate(over="ignore"):
        s = ((mx - mn) / top).astype(np.float16)
    usable = (s > 0) & np.isfinite(s)
    by = np.where(usable, s, np.float16(1)).astype(f)
    z = np.where(usable, np.clip(np.rint(-mn / by), 0, top), f(0))
    q = np.clip(np.rint(y / by[..., None]) + z[..., None], 0, top)
    return np.where(usable[..., None], q, f(0)).astype(np.uint8), s, z.astype(np.uint8)


def pack(codes, bits):
    b = (np.asarray(codes, dtype=np.uint8)[..., None] >> np.arange(bits, dtype=np.uint8)) & 1
    return np.packbits(b.reshape(b.shape[:-2] + (-1,)), axis=-1, bitorder="little")


def unpack(packed, bits):
    b = np.unpackbits(np.asarray(packed, dtype=np.uint8), axis=-1, bitorder="little")
    b = b.reshape(b.shape[:-1] + (-1, bits))
    return (b * (1 << np.arange(bits))).sum(-1).astype(np.uint8)


def parameters(steps, zeros):
    return np.asarray(steps, dtype=np.float16).view(np.uint16).astype(np.uint32) | np.asarray(zeros).astype(np.uint32) << 16


def dequantize(codes, steps, zeros):
    """fp64 values of unpacked codes."""
    return np.asarray(steps, dtype=np.float16).astype(np.float64)[..., None] * (codes.astype(np.float64) - np.asarray(zeros, dtype=np.float64)[..., None])


class Pages:
    """One tensor (keys or values) of a paged cache, on the host."""

    def __init__(self, pages, H, page, bits, fill=0xA5):
        self.page, self.bits = page, bits
        self.codes = np.full((pages, H, page, D * bits // 8), fill, dtype=np.uint8)
        self.params = np.full((pages, H, page), fill * 0x01010101, dtype=np.uint32)      # a negative step and a zero point that is none

    def place(self, table, pos):
        """(page, slot) of a token of the sequence with this table row, or None."""
        if pos < 0 or pos // self.page >= len(table):
            return None
        p = int(table[pos // self.page])
        return (p, pos % self.page) if 0 <= p < self.codes.shape[0] else None

    def write(self, table, pos, row, clip):
        """row fp16 [H, 128]: the token at `pos`."""
        at = self.place(table, pos)
        if at is None:
            return
        q, s, z = grid32(row, clip, self.bits)
        self.codes[at[0], :, at[1]] = pack(q, self.bits)
        self.params[at[0], :, at[1]] = parameters(s, z)

    def values(self, table, positions):
        """fp64 [H, tokens, 128]; zeros where the token has no place."""
        out = np.zeros((self.codes.shape[1], len(positions), D))
        for k, pos in enumerate(positions):
            at = self.place(table, int(pos))
            if at is not None:
                w = self.params[at[0], :, at[1]]
                out[:, k] = dequantize(unpack(self.codes[at[0], :, at[1]], self.bits), (w & 0xFFFF).astype(np.uint16).view(np.float16), w >> 16)
        return out

    def steps(self, table, positions):
        """fp64 [H, tokens]; zeros where the token has no place."""
        out = np.zeros((self.codes.shape[1], len(positions)))
        for k, pos in enumerate(positions):
            at = self.place(table, int(pos))
            if at is not None:
                out[:, k] = (self.params[at[0], :, at[1]] & 0xFFFF).astype(np.uint16).view(np.float16).astype(np.float64)
        return out


def attention64(q, k, v, seen, scale, k_step, v_step, k_bits=4):
    """q [n, 128], k, v [L, 128], seen [n, L], the tokens' steps [L].  Returns out fp64 [n, 128] (zeros for a row that sees nothing) and what the
    bound needs: A [n, 128] = sum_j w_j |v_j|, S [n] = sum_j w_j v_step_j, and the error `delta` [n] of a score:
    s_j (sum_d q_d c_d - z sum_d q_d), each sum fp32 over 128 exact products of at most (2^b - 1) |q_d|, 12 more roundings; and the matrix
    instruction, four of which add a score's products, drops what lies 24 bits below the largest of 33 addends, which counts as max |q| 2^10
    code units of 2^-4 (codes are subnormal numbers there): 4 * 33 * 2^-18 max |q| s_j."""
    q = np.asarray(q, dtype=np.float64)
    n = q.shape[0]
    out, A, S, delta = np.zeros((n, D)), np.zeros((n, D)), np.zeros(n), np.zeros(n)
    for i in range(n):
        j = np.flatnonzero(seen[i])
        if len(j) == 0:
            continue
        s = scale * (k[j] @ q[i])
        w = np.exp(s - s.max())
        w /= w.sum()
        out[i] = w @ v[j]
        A[i] = w @ np.abs(v[j])
        S[i] = w @ v_step[j]
        a = np.abs(q[i])
        delta[i] = abs(scale) * k_step[j].max() * (280 * 2.0 ** -24 * (2 ** k_bits - 1) * a.sum() + 132 * 2.0 ** -18 * a.max())
    return out, A, S, delta


def attention_bound(out, A, S, delta, tokens, v_bits=4):
    """How far an output may be from fp64, from the arithmetic alone.
    scores   off by delta, and 2^-21 from exp2 of a rounded difference: relative errors of the weights
    weights  times the value's step, rounded to fp16: 2^-11 of it (in the subnormals 2^-25 of at least 2^-7 of the row's largest: 2^-32 per token)
    sums     sum_j w_j s_j c_j - sum_j w_j s_j z_j in fp32: at most tokens / 128 + 64 additions behind each other, each 2^-24 of a sum of at most
             (2^b - 1) S; and what the matrix instruction drops of its 33 addends: 33 * 2^-24 of 2^10 code units of 2^-4 of the largest weight
             of its 32 tokens, which sum to S at most over all of them
    output   one rounding to fp16.
    The weights' sum has the relative errors of the scores and sums."""
    top = 2 ** v_bits - 1
    delta = delta[:, None] + 2.0 ** -21
    sums = 2.0 ** -24 * (tokens / 128 + 64)
    return (A * (2.0 ** -11 + 2 * delta + sums) + S[:, None] * (2 * top * sums + top * tokens * 2.0 ** -32 + 33 * 2.0 ** -18)) * (1 + 2.0 ** -8) + \
        np.abs(out) * 2.0 ** -11 + 2.0 ** -24
