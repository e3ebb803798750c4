"""Plain references of the operators on rows: 4-bit floats, head norms with rotary positions, sampling.  Numpy in 64
bits, written from the definitions in include/ssd.h, sharing nothing with the library."""
from __future__ import annotations

import math

import numpy as np

FLOATS4 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def _e4m3_table():
    out = []
    for i in range(127):   # 126 is 448, the largest
        e, m = i >> 3, i & 7
        out.append(m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return np.array(out)


E4M3 = _e4m3_table()


def _nearest(v, table):
    """Values of the table nearest to v, of two as near the one at the even index."""
    i = np.clip(np.searchsorted(table, v), 1, len(table) - 1)
    lo, hi = table[i - 1], table[i]
    up = (v - lo > hi - v) | ((v - lo == hi - v) & (i % 2 == 0))
    return np.where(v >= table[-1], table[-1], np.where(up, hi, lo))


def f4_values(x):
    """x fp32 [rows][k] -> the fp64 values that the packed rows stand for."""
    x = np.asarray(x, np.float64)
    out = np.full(x.shape, np.nan)
    k = x.shape[1]
    for r, row in enumerate(x):
        a = np.abs(row).max()
        if not np.isfinite(a):
            continue
        e = -100
        while a > 2688 * 2.0 ** e:
            e += 1
        y = np.zeros(-(-k // 16) * 16)
        y[:k] = row / 2.0 ** e
        y = y.reshape(-1, 16)
        s = _nearest((np.abs(y).max(1) / 6).astype(np.float32).astype(np.float64), E4M3)
        q = np.divide(np.abs(y), s[:, None], out=np.zeros_like(y), where=s[:, None] > 0)
        c = _nearest(q.astype(np.float32).astype(np.float64), FLOATS4)
        out[r] = (np.sign(y) * c * s[:, None]).reshape(-1)[:k] * 2.0 ** e
    return out


def rotary(x, pos, freq, axis, turn, interleaved=False, gain=None, eps=1e-5):
    """x fp64 [rows][heads][d], pos [rows][axes].  Returns (y, size): size bounds |a| + |b| of each output's pair."""
    x = np.array(x, np.float64)
    if gain is not None:
        x = x / np.sqrt((x * x).mean(2, keepdims=True) + eps) * np.asarray(gain, np.float64)
    y, size = x.copy(), np.abs(x)
    for i in range(turn // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + turn // 2)
        angle = pos[:, axis[i]].astype(np.float64) * freq[i]
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        y[:, :, a], y[:, :, b] = x[:, :, a] * c - x[:, :, b] * s, x[:, :, b] * c + x[:, :, a] * s
        size[:, :, a] = size[:, :, b] = np.abs(x[:, :, a]) + np.abs(x[:, :, b])
    return y, size


def sample(logits, u, temperature, top_k, top_p, min_p):
    """One row, Python floats.  Returns (token, prob)."""
    z = [-math.inf if math.isnan(v) else v for v in map(float, logits)]
    top = max(z)
    if top == -math.inf:
        return -1, 0.0
    order = sorted(range(len(z)), key=lambda i: (-z[i], i))
    if not temperature >= 2.0 ** -100:
        return order[0], 1.0

    def weight(i):
        if z[i] == top:
            return 1.0
        if top == math.inf or z[i] == -math.inf:
            return 0.0
        return math.exp((z[i] - top) / temperature)

    w = [weight(i) for i in order]
    n = len(order) if top_k < 1 else min(top_k, len(order))
    if top_p < 1:
        goal, ahead, m = top_p * math.fsum(w[:n]), 0.0, 0
        while m < n and (m == 0 or ahead < goal):
            ahead += w[m]
            m += 1
        n = m
    if min_p > 0:
        n = max(1, min(n, sum(v >= min_p for v in w)))
    kept = sorted(order[:n])
    mass = [weight(i) for i in kept]
    total, run = math.fsum(mass), 0.0
    for i, m in zip(kept, mass):
        run += m
        if run > u * total:
            return i, m / total
    last = max((i for i, m in zip(kept, mass) if m > 0))
    return last, weight(last) / total
