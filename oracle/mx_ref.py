"""CPU oracle of the operators in 4 bits and with grouped heads (numpy, float64), written from the format's definition in
include/dllava_mx.h; test infrastructure only."""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


# ---- the format -----------------------------------------------------------------------------------------------------------------
def quantize(x):
    """Codes [..., K] and scale bytes [..., K/32] (uint8) of x, blocks of 32 along the last axis."""
    x = np.asarray(x, np.float64)
    b = x.reshape(*x.shape[:-1], -1, 32)
    finite = np.isfinite(b).all(-1)
    amax = np.where(finite, np.abs(np.where(np.isfinite(b), b, 0.0)).max(-1), 1.0)
    m, e = np.frexp(np.where(amax > 0, amax, 2.0 ** -140))  # amax = m 2^e, m in [0.5, 1)
    s = np.clip((e - 1) + (m > 0.875) - 2 + 127, 1, 252)
    a = np.abs(np.where(finite[..., None], b, 0.0)) / np.exp2(s - 127.0)[..., None]
    d = np.abs(a[..., None] - GRID)
    low = d.argmin(-1)                                      # ties: the lower one ...
    up = np.minimum(low + 1, 7)
    tie = (d[..., :] == d.min(-1, keepdims=True)).sum(-1) == 2
    code = np.where(tie & (low % 2 == 1), up, low)          # ... unless its code is odd
    code = np.where(finite[..., None], code, 0) + 8 * np.signbit(b)
    return code.reshape(x.shape).astype(np.uint8), np.where(finite, s, 255).astype(np.uint8)


def dequantize(codes, scales):
    v = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return v * np.repeat(s, 32, -1)


def pack(codes, scales):
    """The bytes of a packed matrix."""
    M, K = codes.shape
    Kp, Mp = -(-K // 512) * 512, -(-M // 16) * 16
    c = np.zeros((M, Kp), np.uint8)
    c[:, :K] = codes
    z = np.full((Mp, Kp // 32), 127, np.uint8)
    z[:M, :K // 32] = scales
    out = np.zeros((Mp // 16, Kp // 512, 4, 16, 4), np.uint8)
    for r in range(Mp):
        for c_ in range(Kp // 32):
            out[r // 16, c_ // 16, c_ % 4, r % 16, c_ % 16 // 4] = z[r, c_]
    return np.concatenate([(c[:, 0::2] | (c[:, 1::2] << 4)).reshape(-1), out.reshape(-1)])


# ---- the paged cache ------------------------------------------------------------------------------------------------------------
class Cache:
    """Pages [n_pages, H, 17 Dh] in 4 bits with their table and lengths."""

    def __init__(self, pages, table, lens):
        self.pages, self.table, self.lens = pages.copy(), np.asarray(table), np.asarray(lens, np.int64).copy()
        self.H, self.Dh = pages.shape[1], pages.shape[2] // 17
        self.cap = 16 * self.table.shape[1]

    def put(self, b, pos, k, v):
        """One token [H, Dh] of sequence b."""
        Dh, blocks, t = self.Dh, self.Dh // 32, pos % 16
        page = self.pages[self.table[b, pos // 16]]
        (kc, ks), (vc, vs) = quantize(k), quantize(v)
        page[:, t * Dh // 2:(t + 1) * Dh // 2] = kc[:, 0::2] | (kc[:, 1::2] << 4)
        for c in range(16):
            for m in range(blocks):
                page[:, 8 * Dh + ((t // 4 * 16 + c) * 4 + t % 4) * blocks + m] = vc[:, 32 * m + c] | (vc[:, 32 * m + 16 + c] << 4)
        page[:, 16 * Dh + t * blocks:16 * Dh + (t + 1) * blocks] = ks
        page[:, 16 * Dh + Dh // 2 + t * blocks:16 * Dh + Dh // 2 + (t + 1) * blocks] = vs

    def get(self, b, pos):
        """K, V [H, Dh] of one token."""
        Dh, blocks, t = self.Dh, self.Dh // 32, pos % 16
        page = self.pages[self.table[b, pos // 16]]
        kb = page[:, t * Dh // 2:(t + 1) * Dh // 2]
        kc = np.stack([kb & 15, kb >> 4], -1).reshape(self.H, Dh)
        vc = np.zeros_like(kc)
        for c in range(16):
            for m in range(blocks):
                byte = page[:, 8 * Dh + ((t // 4 * 16 + c) * 4 + t % 4) * blocks + m]
                vc[:, 32 * m + c], vc[:, 32 * m + 16 + c] = byte & 15, byte >> 4
        ks = page[:, 16 * Dh + t * blocks:16 * Dh + (t + 1) * blocks]
        vs = page[:, 16 * Dh + Dh // 2 + t * blocks:16 * Dh + Dh // 2 + (t + 1) * blocks]
        return dequantize(kc, ks), dequantize(vc, vs)

    def rows(self, b, n):
        """K, V [n, H, Dh] of the first n tokens."""
        if n == 0:
            z = np.zeros((0, self.H, self.Dh))
            return z, z
        got = [self.get(b, t) for t in range(n)]
        return np.stack([g[0] for g in got]), np.stack([g[1] for g in got])


def attention(q, K, V, scale, causal=False):
    """q [m, Hq, Dh], K, V [n, H, Dh]: outputs [m, Hq, Dh], the weighted magnitudes sum_j w_j |v_j| of each, and the largest
    sum |q| |k| * scale per row and head [m, Hq] (what the rounding errors are proportional to)."""
    m, Hq, Dh = q.shape
    n, H, _ = K.shape
    G = Hq // H
    o, mag, big = np.zeros((m, Hq, Dh)), np.zeros((m, Hq, Dh)), np.zeros((m, Hq))
    for h in range(Hq):
        k, v = K[:, h // G], V[:, h // G]
        s = scale * (q[:, h] @ k.T)
        if causal:
            s = np.where(np.arange(n)[None] > np.arange(m)[:, None], -np.inf, s)
        w = np.exp(s - s.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        o[:, h], mag[:, h] = w @ v, w @ np.abs(v)
        big[:, h] = scale * (np.abs(q[:, h]) @ np.abs(k).T).max(-1)
    return o, mag, big


# ---- linear layers --------------------------------------------------------------------------------------------------------------
def linear(x, W, bias, act, residual):
    """y, and what the rounding of its sums is proportional to."""
    from math import erf
    y, mag = x @ W.T, np.abs(x) @ np.abs(W).T
    if bias is not None:
        y, mag = y + bias, mag + np.abs(bias)
    if act == 1:
        y = 0.5 * y * (1.0 + np.vectorize(erf)(y / np.sqrt(2.0)))
        mag = 1.13 * mag                                    # the largest slope of GELU
    if residual is not None:
        if act == 2:
            with np.errstate(over="ignore"):
                gate = residual / (1.0 + np.exp(-residual))
            y, mag = y * gate, mag * np.abs(gate)
        else:
            y, mag = y + residual, mag + np.abs(residual)
    return y, mag
