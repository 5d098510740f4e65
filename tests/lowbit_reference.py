"""Plain implementations of the microscaled 4-bit formats and of the 8-bit key/value cache, on the
host: the roundings that a format defines are taken in the precision it defines them in, products,
sums and softmax in 64 bits."""
from __future__ import annotations

import numpy as np
import torch

E2M1 = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
TOKENS = 16


def round_e2m1(x):
    """Codes 0..15 of fp32 numbers: to nearest, ties to the even code, at most 6."""
    a = np.abs(x).astype(np.float64)
    mids = (E2M1[1:] + E2M1[:-1]) / 2
    up = np.array([False, True, False, True, False, True, False])       # a tie goes up from an odd code
    q = sum(np.where(u, a >= m, a > m).astype(np.int64) for m, u in zip(mids, up))
    return (q + 8 * np.signbit(x)).astype(np.uint8)


def round_e4m3(x):
    """Values of the nearest e4m3 numbers (ties to even), at most 448, of non-NaN numbers."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(x)
    e = np.floor(np.log2(np.maximum(a, 2.0 ** -6)))
    e = np.where(2.0 ** e > np.maximum(a, 2.0 ** -6), e - 1, e)
    ulp = 2.0 ** (e - 3)
    return np.sign(x) * np.minimum(np.rint(a / ulp) * ulp, 448.0)


def e4m3_bytes(v):
    return torch.from_numpy(np.ascontiguousarray(v, dtype=np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


def fp4_quantize(x, fmt, g=None):
    """(codes [rows][padded cols / 2], scale bytes [rows][blocks], block scales as fp32) of fp32 values that are bf16."""
    rows, cols = x.shape
    b = 32 if fmt == "mx" else 16
    v = np.zeros((rows, -(-cols // 32) * 32), dtype=np.float32)
    v[:, :cols] = x
    v = v.reshape(rows, -1, b)
    bad = ~np.isfinite(v).all(-1)
    amax = np.abs(np.where(np.isfinite(v), v, 0)).max(-1).astype(np.float32)
    with np.errstate(all="ignore"):
        if fmt == "mx":
            e = np.where(amax > 0, np.frexp(amax.astype(np.float64))[1] - 1 - 2, -127).clip(-127, 127)
            byte, d = (e + 127).astype(np.uint8), np.ldexp(1.0, e)
            byte[bad] = 255
            q = round_e2m1(np.where(bad[..., None], 0, v.astype(np.float64) / d[..., None]))
        else:
            g = np.float32(1 if g is None else g)
            t = (amax / np.float32(6)) / g
            bad |= ~(g > 0) | ~np.isfinite(t)
            s = round_e4m3(np.where(bad, 0, t)).astype(np.float32)
            byte = e4m3_bytes(s).copy()
            byte[bad] = 0x7f
            d = s * g
            q = round_e2m1(np.where(bad[..., None] | (d[..., None] == 0), np.float32(0), v / d[..., None]))
    d = np.where(bad, np.nan, d)
    q = q.reshape(rows, -1)
    return q[:, ::2] | (q[:, 1::2] << 4), byte, d


def tiled_scales(byte):
    """Scale bytes [rows][blocks] in tiles of 128 rows x 4 blocks."""
    rows, n = byte.shape
    nt = -(-n // 4)
    out = np.zeros(-(-rows // 128) * nt * 512, dtype=np.uint8)
    r, j = np.meshgrid(np.arange(rows), np.arange(n), indexing="ij")
    out[((r // 128) * nt + j // 4) * 512 + 16 * (r % 32) + 4 * (r % 128 // 32) + j % 4] = byte
    return out


def fp4_values(codes, d, cols):
    """fp64 values [rows][cols] of codes and block scales."""
    q = np.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[0], -1)
    v = E2M1[q & 7] * np.where(q > 7, -1.0, 1.0)
    return (v.reshape(len(q), d.shape[1], -1) * d[..., None].astype(np.float64)).reshape(len(q), -1)[:, :cols]


def bf16(x):
    return torch.as_tensor(np.asarray(x, dtype=np.float32)).to(torch.bfloat16).float().numpy()


def bf16_up(x):
    """The smallest bf16 number that is not below x >= 0 (fp32)."""
    u = np.asarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return (((u + 0xffff) >> 16) << 16).astype(np.uint32).view(np.float32)


class Cache:
    """The cache on the host: values of codes (fp32) and scales (fp32 holding bf16), by page."""

    def __init__(self, kind, pages, heads, page, dim, table, rng):
        self.kind, self.page, self.table = kind, page, table
        self.qmax = np.float32(127 if kind == "int8" else 448)
        shape = (pages, heads, page, dim)
        self.code = [self.round(rng.standard_normal(shape).astype(np.float32) * 40) for _ in range(2)]
        self.scale = [bf16(rng.uniform(0.5, 2, (pages, heads, page // TOKENS)) / 64) for _ in range(2)]

    def round(self, x):
        return (np.rint(x).clip(-127, 127) if self.kind == "int8" else round_e4m3(x)).astype(np.float32)

    def append(self, side, x, starts, lens):
        code, scale = self.code[side], self.scale[side]
        for b, ln in enumerate(lens):
            n = starts[b + 1] - starts[b]
            past = ln - n
            for blk in range(past // TOKENS, -(-ln // TOKENS) if n else 0):
                p = np.arange(blk * TOKENS, min(ln, (blk + 1) * TOKENS))
                page, slot = self.table[b, p[0] // self.page], p % self.page
                old = p < past
                new = x[starts[b] + p[~old] - past]                                       # [tokens][heads][dim]
                with np.errstate(all="ignore"):
                    top = np.abs(np.where(np.isfinite(new), new, 0)).max((0, 2))
                    s_old = scale[page, :, slot[0] // TOKENS].copy() if old.any() else np.zeros_like(top)
                    s = np.maximum(s_old, bf16_up(top / self.qmax))
                    held = code[page][:, slot[old]]                                       # [heads][tokens][dim]
                    at = s[:, None, None]
                    q = np.concatenate((np.where(at > 0, held * s_old[:, None, None] / at, 0),
                                        np.where(at > 0, new.transpose(1, 0, 2) / at, 0)), 1)
                    q = np.where(np.isinf(np.concatenate((held, new.transpose(1, 0, 2)), 1)), np.sign(q) * self.qmax, q)
                code[page][:, slot] = self.round(np.nan_to_num(q, nan=0.0, posinf=self.qmax, neginf=-self.qmax))
                scale[page, :, slot[0] // TOKENS] = s

    def values(self, side, b, length):
        """fp64 [heads][length][dim]."""
        p = np.arange(length)
        page, slot = self.table[b, p // self.page], p % self.page
        return (self.code[side][page, :, slot].astype(np.float64) * self.scale[side][page, :, slot // TOKENS][..., None]).transpose(1, 0, 2)

    def device(self, dev):
        """The same cache as tensors of the library."""
        from paper_2602_17698_b200.binding import Kv8Cache
        dt = torch.int8 if self.kind == "int8" else torch.float8_e4m3fn
        k, v = (torch.from_numpy(c).to(dt).to(dev) for c in self.code)
        ks, vs = (torch.from_numpy(s).to(torch.bfloat16).to(dev) for s in self.scale)
        return Kv8Cache(k, v, ks, vs, torch.from_numpy(self.table.astype(np.int32)).to(dev))


def attention(cache, q, starts, lens, scale, window):
    """fp64: out [tokens][query heads][dim], lse, sum of weight x |v|, largest sum of a score's terms'
    magnitudes, and the largest value scale times the sum of the value codes' magnitudes."""
    heads = cache.code[0].shape[1]
    T, hq, d = q.shape
    g = hq // heads
    out, lse = np.zeros((T, hq, d)), np.full((T, hq), -np.inf)
    mag, top, held = np.zeros((T, hq, d)), np.zeros((T, hq)), np.zeros((T, hq, d))
    for b, ln in enumerate(lens):
        n = starts[b + 1] - starts[b]
        if n == 0:
            continue
        k, v = cache.values(0, b, ln), cache.values(1, b, ln)
        pos = np.arange(ln)
        page, slot = cache.table[b, pos // cache.page], pos % cache.page
        code = np.abs(cache.code[1][page, :, slot]).astype(np.float64).transpose(1, 0, 2)
        size = cache.scale[1][page, :, slot // TOKENS].T
        for i in range(n):
            p = ln - n + i
            lo = max(0, p - window + 1) if window else 0
            for h in range(hq):
                qi = q[starts[b] + i, h].astype(np.float64)
                s = k[h // g, lo:p + 1] @ qi * scale
                m = s.max()
                e = np.exp(s - m)
                t = starts[b] + i
                out[t, h] = e @ v[h // g, lo:p + 1] / e.sum()
                mag[t, h] = e @ np.abs(v[h // g, lo:p + 1]) / e.sum()
                lse[t, h] = m + np.log(e.sum())
                held[t, h] = size[h // g, lo:p + 1].max() * code[h // g, lo:p + 1].sum(0)
                top[t, h] = (np.abs(k[h // g, lo:p + 1]) @ np.abs(qi)).max() * abs(scale)
    return out, lse, mag, top, held
