"""Plain references of the low-bit operators: Python loops and numpy, written from the definitions in
include/ssd.h, sharing nothing with the library."""
from __future__ import annotations

import numpy as np

F = np.float32


def plan(length, add, held, free, table, block, max_blocks, rows):
    """One step's plan on Python lists.  free: the free stack (last handed out first).  Returns
    (table, held, free, row_start, slot)."""
    table, held, free = [list(r) for r in table], list(held), list(free)
    for b, l in enumerate(length):
        if l < 0:
            free += table[b][:held[b]]
            held[b] = 0
    row_start, slot = [0], []
    for b, (l, a) in enumerate(zip(length, add)):
        a = 0 if l < 0 else a
        if l >= 0:
            need = min(-(-(l + a) // block), max_blocks)
            for j in range(held[b], need):
                table[b][j] = free[-1] if free else -1
                if free:
                    free.pop()
                    held[b] += 1
        for i in range(a):
            pos = l + i
            j = pos // block
            ok = j < max_blocks and table[b][j] >= 0
            slot.append(table[b][j] * block + pos % block if ok else -1)
        row_start.append(row_start[-1] + a)
    return table, held, free, row_start, slot + [-1] * (rows - len(slot))


class Cache:
    """K or V of one layer: codes [slot][head][dim] and scales [block][head], fp32 arithmetic."""

    def __init__(self, n_blocks, block, heads, dim):
        self.block = block
        self.codes = np.zeros((n_blocks * block, heads, dim), np.int32)
        self.scales = np.zeros((n_blocks, heads), F)

    def append(self, x, slot):
        """x fp32 [rows][heads][dim]."""
        rows = [i for i, s in enumerate(slot) if s >= 0]
        for blk in sorted({slot[i] // self.block for i in rows}):
            mine = [i for i in rows if slot[i] // self.block == blk]
            at = [slot[i] for i in mine]
            first = min(at) % self.block
            new = x[mine].astype(F)
            finite = np.where(np.isfinite(new), np.abs(new), F(0))
            old = self.scales[blk].copy() if first else np.zeros_like(self.scales[blk])
            s = np.maximum(old, np.maximum(finite.max((0, 2)) / F(127), F(2.0 ** -100))).astype(F)
            lo = blk * self.block
            for h in range(len(s)):
                if first and s[h] > old[h]:
                    ratio = F(old[h] / s[h])
                    self.codes[lo:lo + first, h] = np.rint(self.codes[lo:lo + first, h].astype(F) * ratio)
                with np.errstate(invalid="ignore", over="ignore"):
                    q = np.rint(new[:, h] * F(F(1) / s[h]))
                q = np.where(np.isnan(new[:, h]), 0, np.clip(q, -127, 127))
                self.codes[at, h] = q.astype(np.int32)
            self.scales[blk] = s

    def values(self, slot):
        """fp32 values at the slots, zeros where negative."""
        slot = np.asarray(slot)
        v = self.codes[np.maximum(slot, 0)].astype(F) * self.scales[np.maximum(slot, 0) // self.block][:, :, None]
        return np.where((slot >= 0)[:, None, None], v, F(0)).astype(F)


def attention(q, kv_of, length, add, heads, kv_heads, scale, masks=None):
    """64-bit attention of ragged rows.  q [rows][heads][dim]; kv_of(b) -> (k, v, present, s) of request b's
    tokens: [n][kv_heads][dim] each, a bool [n] and v's scales [n][kv_heads].  Returns (o, weight, size, floor):
    o, sum_j p_j |v_j|, the largest scale * sum_d |q_d k_jd| of each (row, head), and
    max_j(p_j s_j) * sum_j |c_j| for v_j = c_j s_j."""
    group = heads // kv_heads
    o = np.zeros(q.shape)
    weight = np.zeros(q.shape)
    floor = np.zeros(q.shape)
    size = np.zeros(q.shape[:2])
    r = 0
    for b, (l, a) in enumerate(zip(length, add)):
        if l < 0 or a == 0:
            continue
        k, v, present, sv = kv_of(b)
        for i in range(a):
            seen = present.copy()
            for j in range(a):
                if l + j < len(seen):
                    seen[l + j] &= bool(masks[r] >> j & 1) if masks is not None else j <= i
            idx = np.nonzero(seen)[0]
            for h in range(heads) if len(idx) else ():
                kk, vv = k[idx, h // group].astype(np.float64), v[idx, h // group].astype(np.float64)
                qq = q[r, h].astype(np.float64)
                s = scale * (kk @ qq)
                p = np.exp(s - s.max())
                p /= p.sum()
                o[r, h] = p @ vv
                weight[r, h] = p @ np.abs(vv)
                ss = sv[idx, h // group].astype(np.float64)
                floor[r, h] = (p * ss).max() * (np.abs(vv) / ss[:, None]).sum(0)
                size[r, h] = scale * (np.abs(kk) @ np.abs(qq)).max()
            r += 1
    return o, weight, size, floor


def bf16_round(x):
    """fp32 array rounded to bf16 (nearest even), as fp32."""
    u = np.asarray(x, F).view(np.uint32).astype(np.uint64)
    return ((u + 0x7fff + (u >> 16 & 1)) & 0xffff0000).astype(np.uint32).view(F)


def quantize4(w, group):
    """fp32 weights [n][k] -> the fp32 values their 4-bit codes stand for."""
    n, k = w.shape
    pad = np.zeros((n, -(-k // group) * group), F)
    pad[:, :k] = w
    g = pad.reshape(n, -1, group)
    s = bf16_round(np.abs(g).max(2) / F(7))
    inv = np.divide(F(1), s, out=np.zeros_like(s), where=s > 0)
    c = np.clip(np.rint(g * inv[:, :, None]), -8, 7).astype(F)
    return (c * s[:, :, None]).reshape(n, -1)[:, :k]
