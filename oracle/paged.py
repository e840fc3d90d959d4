"""CPU float64 oracle for rotary positions and the paged key/value cache.

TEST INFRASTRUCTURE ONLY (see oracle.naive): the plain definitions the HIP kernels are
checked against, in NumPy, one row at a time. Nothing here is shared with the GPU path.

Rotation. Pair i of a row at position p, (x_i, x_{i+r/2}) or interleaved
(x_{2i}, x_{2i+1}), as a complex number, times a e^{i p f_i}; columns from r on stay.

4-bit rows. Per 32 columns the smallest 2^e, e >= -125, with all magnitudes below
7 2^e, each value the nearest of +-{0, .5, 1, 1.5, 2, 3, 4, 6} 2^e below 2^128, ties to
the code with an even number; NaN throughout if one of them is not finite.

Pages. Token p of sequence b is row p % page of page table[b, p // page]; a number that
is no page holds nothing.
"""
from __future__ import annotations

import numpy as np

__all__ = ["rotate", "CODES", "to_codes", "from_codes", "Cache"]

CODES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def rotate(x, pos, freqs, amplitude=1.0, interleaved=False, back=False):
    """x [..., d] (float64) with positions pos [...]; back: the transposed map."""
    x = np.array(x, dtype=np.float64)
    freqs = np.asarray(freqs, dtype=np.float64)
    r = 2 * len(freqs)
    angle = np.asarray(pos, dtype=np.float64)[..., None] * freqs
    u = x[..., 0:r:2] if interleaved else x[..., :r // 2]
    w = x[..., 1:r:2] if interleaved else x[..., r // 2:r]
    z = (u + 1j * w) * (amplitude * np.exp((-1j if back else 1j) * angle))
    y = x.copy()
    if interleaved:
        y[..., 0:r:2], y[..., 1:r:2] = z.real, z.imag
    else:
        y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
    return y


def to_codes(x):
    """x [..., d] -> (bytes [..., d/2], scales [..., d/32])."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(-1, 32)
    codes = np.zeros((len(g), 32), dtype=np.uint8)
    scales = np.zeros(len(g), dtype=np.uint8)
    for i, v in enumerate(g):
        if not np.all(np.isfinite(v)):
            scales[i] = 255
            continue
        e = -125
        while np.abs(v).max() >= 7 * 2.0 ** e:
            e += 1
        scales[i] = e + 127
        off = np.abs(np.abs(v)[:, None] / 2.0 ** e - CODES)
        off[:, CODES * 2.0 ** e >= 2.0 ** 128] = np.inf
        best = off.min(1)
        for j in range(32):
            near = np.flatnonzero(off[j] == best[j])
            code = near[0] if len(near) == 1 else near[near % 2 == 0][0]
            codes[i, j] = code + (8 if v[j] < 0 else 0)
    codes = codes.reshape(x.shape)
    return codes[..., 0::2] | (codes[..., 1::2] << 4), scales.reshape(x.shape[:-1] + (x.shape[-1] // 32,))


def from_codes(codes, scales):
    codes = np.asarray(codes, dtype=np.uint8)
    both = np.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[:-1] + (-1,))
    v = np.where(both & 8, -1.0, 1.0) * CODES[both & 7]
    unit = np.where(np.asarray(scales) == 255, np.nan, 2.0 ** (np.asarray(scales, dtype=np.float64) - 127))
    return v * np.repeat(unit, 32, -1)


class Cache:
    """A pool (float64 values [num_pages, Hkv, page, d]) and its tables."""

    def __init__(self, k_pages, v_pages, table):
        self.k, self.v = np.array(k_pages, dtype=np.float64), np.array(v_pages, dtype=np.float64)
        self.table = np.asarray(table)
        self.page = self.k.shape[2]

    def place(self, b, p):
        """(page, row) of token p of sequence b, or None."""
        if p < 0 or p // self.page >= self.table.shape[1]:
            return None
        at = int(self.table[b, p // self.page])
        return (at, p % self.page) if 0 <= at < len(self.k) else None

    def write(self, b, p, k, v):
        """k, v [Hkv, d] as they are stored."""
        at = self.place(b, p)
        if at is not None:
            self.k[at[0], :, at[1]], self.v[at[0], :, at[1]] = k, v

    def rows(self, b, tokens):
        """The tokens (indices) that exist, K and V [Hkv, T, d] of them."""
        at = [(p, self.place(b, p)) for p in tokens]
        at = [(p, x) for p, x in at if x is not None]
        pages, rows = np.array([x[0] for _, x in at], dtype=int), np.array([x[1] for _, x in at], dtype=int)
        return [p for p, _ in at], self.k[pages, :, rows].transpose(1, 0, 2), self.v[pages, :, rows].transpose(1, 0, 2)

    def attend(self, q, T, scale):
        """q [B, Hq, d], the first T[b] tokens: (O, L), and the sum of p |v| per
        output and the largest sum of |q k| scale per (b, h), for error bounds."""
        B, Hq, d = q.shape
        G = Hq // self.k.shape[1]
        O, A = np.zeros((B, Hq, d)), np.zeros((B, Hq, d))
        L, S = np.full((B, Hq), -np.inf), np.zeros((B, Hq))
        for b in range(B):
            _, K, V = self.rows(b, range(int(T[b])))
            for h in range(Hq):
                if K.shape[1] == 0:
                    continue
                s = scale * (K[h // G] @ q[b, h])
                m = s.max()
                e = np.exp(s - m)
                L[b, h] = m + np.log(e.sum())
                O[b, h] = e @ V[h // G] / e.sum()
                A[b, h] = e @ np.abs(V[h // G]) / e.sum()
                S[b, h] = abs(scale) * (np.abs(K[h // G]) @ np.abs(q[b, h])).max()
        return O, L, A, S
