"""Plain binary64 / integer references for the serving operators: microscaled 4-bit weights and
the 8-bit key/value cache.  Written from the formats' definitions; shares nothing with the library."""
import math

import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


# ------------------------------------------------------------------ microscaled 4-bit

def mx4_quantize(x: torch.Tensor):
    """(codes int [rows, blocks, 32], scale bytes int [rows, blocks]) of a real matrix."""
    w = x.detach().cpu().double().numpy()
    rows, cols = w.shape
    nb = (cols + 31) // 32
    p = np.zeros((rows, nb * 32))
    p[:, :cols] = w
    p = p.reshape(rows, nb, 32)
    bad = ~np.isfinite(p).all(-1)
    p = np.where(bad[..., None], 0.0, p)
    amax = np.abs(p).max(-1)
    _, e = np.frexp(amax)                                   # amax = m 2^e, m in [1/2, 1)
    e = np.where(amax > 0, np.maximum(e - 3, -127), -127)
    a = np.abs(p) / np.ldexp(1.0, e)[..., None]
    dist = np.abs(a[..., None] - GRID)
    dist[..., 1::2] += 1e-9                                 # a tie goes to the even code
    code = dist.argmin(-1) + 8 * np.signbit(p)
    code[bad] = 0
    return code, np.where(bad, 255, e + 127)


def mx4_values(code, byte):
    v = np.where(code >= 8, -1.0, 1.0) * GRID[code & 7] * np.ldexp(1.0, byte - 127)[..., None]
    v[byte == 255] = np.nan
    return v.reshape(code.shape[0], -1)


def mx4_pack(code, byte):
    """The stored codes and the tiled scale bytes."""
    rows, nb = byte.shape
    pairs = code.reshape(rows, nb * 16, 2)
    codes = (pairs[..., 0] | (pairs[..., 1] << 4)).astype(np.uint8)
    kt = (nb + 3) // 4
    scales = np.zeros((rows + 127) // 128 * kt * 512, dtype=np.uint8)
    r, b = np.arange(rows)[:, None], np.arange(nb)[None]
    scales[(r // 128 * kt + b // 4) * 512 + r % 32 * 16 + r // 32 % 4 * 4 + b % 4] = byte
    return codes, scales


def mx4_random(rows, cols, seed, scale=0.02, dtype=torch.bfloat16):
    """A random pruned matrix in 4 bits: (codes, scales, binary64 values)."""
    g = torch.Generator().manual_seed(seed)
    w = (torch.randn(rows, cols, generator=g) * scale * (torch.rand(rows, cols, generator=g) < 0.5)).to(dtype)
    code, byte = mx4_quantize(w)
    codes, scales = mx4_pack(code, byte)
    return torch.from_numpy(codes), torch.from_numpy(scales), torch.from_numpy(mx4_values(code, byte)[:, :cols])


# ------------------------------------------------------------------ 8-bit cache

def e4m3(x: np.ndarray):
    """Nearest e4m3 value (ties to even) of |x| <= 448; what is not finite becomes NaN."""
    with np.errstate(invalid="ignore"):
        a = np.abs(x)
        _, e = np.frexp(np.where(np.isfinite(a), a, 0.0))
        step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
        y = np.round(a / step) * step
        return np.where(np.isfinite(x), np.copysign(y, x), np.nan)


def cache_exponent(amax: float) -> int:
    e = -126
    if amax > 0:
        m, x = math.frexp(amax)
        e = max(-126, x - 9 + (m > 0.875))
    return e


def finite_amax(x: np.ndarray) -> float:
    a = np.abs(x[np.isfinite(x)])
    return float(a.max()) if a.size else 0.0


class PlainCache:
    """The cache's contents as binary64 code values and exponents."""

    def __init__(self, cache):
        self.k = cache.k.cpu().view(torch.float8_e4m3fn).double().numpy().copy()
        self.v = cache.v.cpu().view(torch.float8_e4m3fn).double().numpy().copy()
        self.ke = np.round(np.log2(cache.k_scale.cpu().double().numpy())).astype(int)
        self.ve = np.round(np.log2(cache.v_scale.cpu().double().numpy())).astype(int)
        self.table = cache.table.cpu().numpy()
        self.T = cache.block_tokens

    def block(self, seq, place):
        if place >= self.table.shape[1]:
            return -1
        b = int(self.table[seq, place])
        return b if 0 <= b < self.k.shape[0] else -1

    def append(self, K, V, start, count=None):
        for x, codes, exps in ((K, self.k, self.ke), (V, self.v, self.ve)):
            x = x.detach().cpu().double().numpy()
            for b in range(x.shape[0]):
                n = x.shape[1] if count is None else min(int(count[b]), x.shape[1])
                s = int(start[b])
                if s < 0 or n <= 0:
                    continue
                for place in range(s // self.T, (s + n - 1) // self.T + 1):
                    blk = self.block(b, place)
                    if blk < 0:
                        continue
                    lo, hi = max(s, place * self.T), min(s + n, (place + 1) * self.T)
                    for h in range(x.shape[2]):
                        new = x[b, lo - s:hi - s, h]
                        e = cache_exponent(finite_amax(new))
                        old = lo - place * self.T
                        if old > 0:
                            e = max(e, int(exps[blk, h]))
                            codes[blk, h, :old] = e4m3(codes[blk, h, :old] * 2.0 ** (int(exps[blk, h]) - e))
                        codes[blk, h, old:old + hi - lo] = e4m3(new / 2.0 ** e)
                        exps[blk, h] = e

    def dense(self, which, seq, head, n):
        """[n, head size] values of the first n tokens; None rows where no block is named."""
        codes, exps = (self.k, self.ke) if which == "k" else (self.v, self.ve)
        out = np.zeros((n, codes.shape[3]))
        here = np.zeros(n, dtype=bool)
        for j in range(n):
            b = self.block(seq, j // self.T)
            if b >= 0:
                out[j] = codes[b, head, j % self.T] * 2.0 ** int(exps[b, head])
                here[j] = True
        return out, here

    def attention(self, Q, lens, max_len, scale, acc_in=None):
        """(O, lse, acc) in binary64, and for error bounds the weighted magnitudes of the values
        [like O] and the largest sum of magnitudes behind a score [like lse]."""
        Q = Q.detach().cpu().double().numpy()
        B, n, Hq, D = Q.shape
        H = self.k.shape[1]
        G = Hq // H
        O, lse = np.zeros(Q.shape), np.full((B, n, Hq), -np.inf)
        acc = np.zeros((B, H, max_len))
        mag, terms = np.zeros(Q.shape), np.zeros((B, n, Hq))
        cap = self.table.shape[1] * self.T
        for b in range(B):
            length = int(lens[b])
            stored = max(0, min(length, max_len, cap))
            for h in range(H):
                K, here = self.dense("k", b, h, stored)
                V, _ = self.dense("v", b, h, stored)
                if acc_in is not None:
                    old = max(0, min(stored, length - n))
                    acc[b, h, :old] = acc_in[b, h, :old]
                for i in range(n):
                    see = here & (np.arange(stored) <= length - n + i)
                    if not see.any():
                        continue
                    for x in range(G):
                        s = (K[see] @ Q[b, i, h * G + x]) * scale
                        p = np.exp(s - s.max())
                        lse[b, i, h * G + x] = s.max() + math.log(p.sum()) if np.isfinite(p.sum()) else np.nan
                        p /= p.sum()
                        O[b, i, h * G + x] = p @ V[see]
                        mag[b, i, h * G + x] = p @ np.abs(V[see])
                        terms[b, i, h * G + x] = (np.abs(K[see]) @ np.abs(Q[b, i, h * G + x])).max() * scale
                        acc[b, h, :stored][see] += p
        return O, lse, acc, mag, terms

    def evict(self, dst, lens, max_len, acc, budget, recent):
        """kept [B, H, budget] and the new contents laid into dst (a PlainCache)."""
        B, H = acc.shape[:2]
        kept = np.full((B, H, budget), -1)
        for b in range(B):
            n = max(0, min(int(lens[b]), max_len, self.table.shape[1] * self.T))
            m = min(n, budget)
            last = min(recent, m)
            for h in range(H):
                a = [math.inf if math.isnan(v) else float(v) for v in acc[b, h, :n - last]]
                nan = [math.isnan(v) for v in acc[b, h, :n - last]]
                best = sorted(range(n - last), key=lambda j: (not nan[j], -a[j], j))[:m - last]
                kept[b, h, :m] = sorted(best) + list(range(n - last, n))
                for which, codes, exps in (("k", dst.k, dst.ke), ("v", dst.v, dst.ve)):
                    x, _ = self.dense(which, b, h, n)
                    x = x[kept[b, h, :m]]
                    for place in range((budget + self.T - 1) // self.T):
                        blk = dst.block(b, place)
                        if blk < 0:
                            continue
                        part = np.zeros((self.T, x.shape[1]))
                        piece = x[place * self.T:(place + 1) * self.T]
                        part[:len(piece)] = piece
                        e = cache_exponent(finite_amax(part))
                        codes[blk, h] = e4m3(part / 2.0 ** e)
                        exps[blk, h] = e
        return kept
