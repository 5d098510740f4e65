"""Plain implementations, on the host in 64 bits, of the 4-bit key/value cache, rotary positions and low-rank adapters."""
from __future__ import annotations

import numpy as np
import torch

from lowbit_reference import E2M1, bf16, e4m3_bytes, round_e2m1, round_e4m3

BLOCK = 16


class Cache4:
    """The cache on the host: codes 0..15, block scales and head scales (fp32), by page."""

    def __init__(self, pages, heads, page, dim, table, rng, head_scales=True):
        self.page, self.table, self.dim = page, table, dim
        shape = (pages, heads, page, dim)
        self.code = [rng.integers(0, 16, shape).astype(np.uint8) for _ in range(2)]
        self.scale = [round_e4m3(np.exp(0.7 * rng.standard_normal((*shape[:3], dim // BLOCK)))).astype(np.float32) for _ in range(2)]
        self.head = [(np.exp2(rng.integers(-3, 3, heads)) * (1 if i else 1.25)).astype(np.float32) if head_scales else np.ones(heads, np.float32)
                     for i in range(2)]
        self.head_scales = head_scales

    def append(self, side, x, starts, lens):
        for b, ln in enumerate(lens):
            n = starts[b + 1] - starts[b]
            p = np.arange(ln - n, ln)
            v = x[starts[b]:starts[b + 1]].astype(np.float32)                             # [tokens][heads][dim]
            v = v.reshape(*v.shape[:2], v.shape[2] // BLOCK, BLOCK)
            g = self.head[side][:, None]
            with np.errstate(all="ignore"):
                amax = np.abs(np.where(np.isfinite(v), v, 0)).max(-1).astype(np.float32)
                t = (amax / np.float32(6)) / g
                good = (g > 0) & np.isfinite(g)
                s = round_e4m3(np.where(good, np.minimum(t, np.float32(448)), 0)).astype(np.float32)
                d = (s * np.where(good, g, 0))[..., None]
                q = np.where(d > 0, v / d, np.float32(0))
                q = np.where(np.isinf(v) & good[..., None], np.copysign(np.float32(6), v), q)
            q = np.nan_to_num(q, nan=0.0, posinf=6.0, neginf=-6.0)
            page, slot = self.table[b, p // self.page], p % self.page
            self.code[side][page, :, slot] = round_e2m1(q).reshape(n, v.shape[1], self.dim)
            self.scale[side][page, :, slot] = s

    def values(self, side, b, length):
        """fp64 [heads][length][dim]."""
        p = np.arange(length)
        page, slot = self.table[b, p // self.page], p % self.page
        q = self.code[side][page, :, slot]
        v = E2M1[q & 7] * np.where(q > 7, -1.0, 1.0)
        s = self.scale[side][page, :, slot].astype(np.float64) * self.head[side].astype(np.float64)[:, None]
        return (v.reshape(*s.shape, BLOCK) * s[..., None]).reshape(v.shape).transpose(1, 0, 2)

    def bytes(self, side):
        """Codes and scales as the library holds them."""
        q = np.zeros((*self.code[side].shape[:3], -(-self.dim // 32) * 32), dtype=np.uint8)
        q[..., :self.dim] = self.code[side]
        s = np.zeros((*self.scale[side].shape[:3], -(-self.dim // 64) * 4), dtype=np.uint8)
        s[..., :self.dim // BLOCK] = e4m3_bytes(self.scale[side])
        return q[..., ::2] | (q[..., 1::2] << 4), s

    def device(self, dev):
        from paper_2602_17698_b200.binding import Kv4Cache
        (k, ks), (v, vs) = ([torch.from_numpy(t).to(dev) for t in self.bytes(side)] for side in range(2))
        heads = [torch.from_numpy(h).to(dev) for h in self.head] if self.head_scales else [None, None]
        return Kv4Cache(k, v, ks, vs, torch.from_numpy(self.table.astype(np.int32)).to(dev), self.dim, *heads)


def attention(cache, q, starts, lens, scale, window):
    """fp64: out [tokens][query heads][dim], lse, sum of weight x |v|, largest sum of a score's terms' magnitudes, and the sum of |v|
    over the keys that a query sees."""
    heads = cache.code[0].shape[1]
    T, hq, d = q.shape
    g = hq // heads
    out, lse, mag, top, held = np.zeros((T, hq, d)), np.full((T, hq), -np.inf), np.zeros((T, hq, d)), np.zeros((T, hq)), np.zeros((T, hq, d))
    for b, ln in enumerate(lens):
        n = starts[b + 1] - starts[b]
        if n == 0:
            continue
        k, v = cache.values(0, b, ln), cache.values(1, b, ln)
        for i in range(n):
            p, t = ln - n + i, starts[b] + i
            lo = max(0, p - window + 1) if window else 0
            for h in range(hq):
                kk, vv, qi = k[h // g, lo:p + 1], v[h // g, lo:p + 1], q[t, h].astype(np.float64)
                s = kk @ qi * scale
                e = np.exp(s - s.max())
                out[t, h] = e @ vv / e.sum()
                mag[t, h] = e @ np.abs(vv) / e.sum()
                held[t, h] = np.abs(vv).sum(0)
                lse[t, h] = s.max() + np.log(e.sum())
                top[t, h] = (np.abs(kk) @ np.abs(qi)).max() * abs(scale)
    return out, lse, mag, top, held


def rotary(x, pos, freq, interleaved, factor=1.0, inverse=False):
    """fp64 of [rows][heads][dim] numbers at integer positions; and the size of a result's two terms."""
    x = np.asarray(x, dtype=np.float64)
    half = len(freq)
    a = np.asarray(pos, dtype=np.longdouble)[:, None] * freq.astype(np.longdouble) * (-1 if inverse else 1)
    c, s = ((f(a) * factor).astype(np.float64)[:, None] for f in (np.cos, np.sin))
    i, j = (np.arange(0, 2 * half, 2), np.arange(1, 2 * half, 2)) if interleaved else (np.arange(half), np.arange(half, 2 * half))
    y, size = x.copy(), np.zeros_like(x)
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    size[..., i] = size[..., j] = (np.abs(x[..., i]) + np.abs(x[..., j])) * abs(factor)
    return y, size


def lora(x, base, a, b, scale, ids, starts):
    """fp64 result, and sums of magnitudes: of the second product's terms, and with the first's terms in their place."""
    x, y = np.asarray(x, dtype=np.float64), np.asarray(base, dtype=np.float64).copy()
    second, first = np.zeros_like(y), np.zeros_like(y)
    for r, i in enumerate(ids):
        rows = slice(starts[r], starts[r + 1])
        if i < 0 or starts[r + 1] == starts[r]:
            continue
        A, B, f = a[i].astype(np.float64), b[i].astype(np.float64), 1.0 if scale is None else float(scale[i])
        h = x[rows] @ A.T
        y[rows] += f * (h @ B.T)
        second[rows] = abs(f) * (np.abs(h) @ np.abs(B).T)
        first[rows] = abs(f) * (np.abs(x[rows]) @ np.abs(A).T @ np.abs(B).T)
    return y, second, first
