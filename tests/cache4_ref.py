"""Plain numpy form of the paged 4-bit cache (include/hqmq_cache4.h): quantisation, the pages' layout and causal attention in
64 bits, element by element and independent of the library."""
from __future__ import annotations

import math

import numpy as np

FLOAT, INT = 0, 1
LARGEST = 49152.0
GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def width_of(D):
    return -(-D // 32) * 32 if D <= 128 else -(-D // 64) * 64


def scale_bytes(fmt):
    return 1 if fmt == FLOAT else 4


def half_of(x):
    """fp64 -> the nearest fp16 (numpy rounds once), as fp64."""
    with np.errstate(over="ignore"):
        return np.asarray(x, np.float64).astype(np.float16).astype(np.float64)


def quantise(fmt, x):
    """x: fp64 [..., D] (NaN as 0).  codes uint8 [..., width], scales uint8 [..., G, 1 or 4]."""
    x = np.clip(np.nan_to_num(np.asarray(x, np.float64), nan=0.0, posinf=np.inf, neginf=-np.inf), -LARGEST, LARGEST)
    D = x.shape[-1]
    W = width_of(D)
    codes = np.zeros(x.shape[:-1] + (W,), np.uint8)
    scales = np.zeros(x.shape[:-1] + (W // 32, scale_bytes(fmt)), np.uint8)
    for g in range(W // 32):
        v = x[..., 32 * g:min(32 * g + 32, D)]
        if fmt == FLOAT:
            top = np.abs(v).max(-1) if v.shape[-1] else np.zeros(x.shape[:-1])
            e = np.full(top.shape, -23)
            for k in range(-23, 13):
                e = np.where(top > 7.0 * 2.0 ** k, k + 1, e)
            y = v / (2.0 ** e)[..., None]
            gap = np.abs(np.abs(y)[..., None] - GRID)
            tie = gap == gap.min(-1, keepdims=True)
            even = tie & (np.arange(8) % 2 == 0)
            pick = np.where(even.any(-1), even.argmax(-1), tie.argmax(-1))
            codes[..., 32 * g:32 * g + v.shape[-1]] = pick | (np.signbit(v) << 3)
            scales[..., g, 0] = e + 127
            continue
        if not v.shape[-1]:
            continue
        low, high = v.min(-1), v.max(-1)
        step = ((high - low).astype(np.float32) * np.float32(1 / 15)).astype(np.float16)
        least = low.astype(np.float16)
        s = step.astype(np.float64)[..., None]
        q = np.divide(v - least.astype(np.float64)[..., None], s, out=np.zeros_like(v), where=s > 0)
        codes[..., 32 * g:32 * g + v.shape[-1]] = np.clip(np.rint(q), 0, 15)
        scales[..., g, :] = np.stack([step, least], -1).view(np.uint8).reshape(*step.shape, 4)
    return codes, scales


def dequantise(fmt, codes, scales, D):
    """fp64 values [..., D]."""
    c = codes.reshape(*codes.shape[:-1], -1, 32).astype(np.int64)
    if fmt == FLOAT:
        y = GRID[c & 7] * np.where(c & 8, -1.0, 1.0) * 2.0 ** (scales.astype(np.float64) - 127)
    else:
        pair = np.ascontiguousarray(scales).view(np.float16).astype(np.float64)
        y = half_of(pair[..., 1:] + c * pair[..., :1])
    return y.reshape(codes.shape)[..., :D]


def parts(W):
    out, at = [], 0
    for w in (128, 64, 32):
        while W - at >= w:
            out.append((at, w))
            at += w
    return out


class Pages:
    """The four buffers as numpy byte arrays."""

    def __init__(self, n_pages, page, H, D, fmt, fill=0):
        self.n_pages, self.page, self.H, self.D, self.fmt = n_pages, page, H, D, fmt
        self.W = width_of(D)
        n = scale_bytes(fmt)
        self.k = np.full((n_pages, H, page, self.W // 2), fill, np.uint8)
        self.v = np.full((n_pages, H, page // 4, 2 * self.W), fill, np.uint8)
        self.ks = np.full((n_pages, H, page, self.W // 32, n), fill, np.uint8)
        self.vs = np.full((n_pages, H, page // 4, self.W // 32, 4, n), fill, np.uint8)

    def _v_bytes(self, t):
        """Index of every byte (channel pair) of token t in its block of four."""
        at, run, base = np.zeros(self.W // 2, np.int64), 0, 0
        for first, w in parts(self.W):
            run = w // 32  # bytes of a run
            i = np.arange(w // 2)
            at[first // 2:(first + w) // 2] = base + i // run * 4 * run + t % 4 * run + i % run
            base += 2 * w
        return at

    def put(self, role, page, slot, codes, scales):
        """codes [H, W], scales [H, G, n] of one token."""
        both = codes[:, 0::2] | codes[:, 1::2] << 4
        if role == 0:
            self.k[page, :, slot], self.ks[page, :, slot] = both, scales
        else:
            self.v[page, :, slot // 4][:, self._v_bytes(slot)] = both
            self.vs[page, :, slot // 4, :, slot % 4] = scales

    def get(self, role, page, slot):
        if role == 0:
            both, scales = self.k[page, :, slot], self.ks[page, :, slot]
        else:
            both, scales = self.v[page, :, slot // 4][:, self._v_bytes(slot)], self.vs[page, :, slot // 4, :, slot % 4]
        codes = np.stack([both & 15, both >> 4], -1).reshape(self.H, self.W)
        return dequantise(self.fmt, codes, scales, self.D)

    def sequence(self, role, table, length):
        """fp64 [length, H, D] and which tokens there are (their page is one)."""
        out, there = np.zeros((length, self.H, self.D)), np.zeros(length, bool)
        for t in range(length):
            p = int(table[t // self.page])
            if 0 <= p < self.n_pages:
                out[t], there[t] = self.get(role, p, t % self.page), True
        return out, there


def attend(q, k, v, there, pos, scale, window, half, weight):
    """q [rows, Hq, D] at positions pos, k and v [length, H, D].  o, lse and bounds on the errors of both.

    half: half a step of the result's type relative to a value; weight: that of a weight.  A score is a sum of D exact products
    in fp32 (each addition off by at most 2^-23, truncation included) times scale * log2 e (two roundings) minus a reference
    (one).  A weight is off by its exponent's error, 2^-22 of the exponential, its rounding, and as far as it is tiny beside the largest, 2^-31
    of that one: weights are kept 2^7 or more above fp16's last bit 2^-24 (2^-25 half of it), the reference staying within 2^22 of the
    largest.  Sums over n tokens lose at most n 2^-23 of the sum of magnitudes, rescalings 2^-22 each: at most one for every 32 tokens."""
    rows, Hq, D = q.shape
    n, H = k.shape[:2]
    o, lse = np.zeros(q.shape), np.full((rows, Hq), -np.inf)
    tol, tol_lse = np.zeros(q.shape), np.zeros((rows, Hq))
    for r in range(rows):
        t = np.arange(n)
        seen = (t <= pos[r]) & there
        if window:
            seen &= t > pos[r] - window
        if not seen.any():
            continue
        for hq in range(Hq):
            h = hq // (Hq // H)
            K, V = k[seen, h], v[seen, h]
            s = scale * (K @ q[r, hq])
            size = abs(scale) * (np.abs(K) @ np.abs(q[r, hq]))
            M = s.max()
            w = np.exp(s - M)
            L = w.sum()
            o[r, hq], lse[r, hq] = w @ V / L, M + math.log(L)
            m = int(seen.sum())
            exponent = (D + 2) * 2.0 ** -23 * size + 2.0 ** -22 * np.abs(s - M) + 2.0 ** -22 * abs(M)
            sums = (m + m / 32 + 64) * 2.0 ** -23
            common = exponent.max() + 2.0 ** -21 + sums
            tiny = 2.0 ** -31
            mean = w @ np.abs(V) / L
            tol[r, hq] = (2 * common + 2 * weight) * mean + 2 * tiny * np.abs(V).sum(0) / L + half * np.abs(o[r, hq]) + 2.0 ** -25
            tol_lse[r, hq] = common + tiny * m / L + 2.0 ** -22 * abs(lse[r, hq]) + 2.0 ** -20
    return o, lse, tol, tol_lse
