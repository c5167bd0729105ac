"""The microscaled formats and operators of include/sjd.h in 64 bits on the CPU, element by element from their definitions."""
import math

import numpy as np

LARGEST = {8: 448.0, 4: 6.0}


def table(bits):
    """value of every code"""
    if bits == 4:
        half = [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    else:
        half = [math.ldexp(8 + m, e - 10) if e else math.ldexp(m, -9) for e in range(16) for m in range(8)]
        half[127] = math.nan
    return np.array(half + [-x for x in half])


def step(y, bits):
    """distance of neighbouring values of the format at |y|"""
    e = np.floor(np.log2(np.maximum(np.abs(y), 1e-300)))
    return 2.0 ** (np.maximum(e, -6) - 3) if bits == 8 else 2.0 ** (np.maximum(e, 0) - 1)


def scale_byte(amax, bits):
    byte = 0
    while amax > LARGEST[bits] * 2.0 ** (byte - 127):
        byte += 1
    return byte


def scale_bytes(amax, bits):
    """the same for an array: exponents by frexp, amax = m 2^e with 0.5 <= m < 1"""
    m, e = np.frexp(amax)
    top, half = (9, 0.875) if bits == 8 else (3, 0.75)
    return np.where(amax > 0, np.maximum(e - top + (m > half) + 127, 0), 0).astype(np.int64)


def nearest(y, bits):
    """codes nearest to y, |y| <= the largest; ties to the even code"""
    vals = table(bits)[: 127 if bits == 8 else 8]
    a = np.abs(y)
    hi = np.clip(np.searchsorted(vals, a), 1, len(vals) - 1)
    lo = hi - 1
    dl, dh = a - vals[lo], vals[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return (code + np.where(np.signbit(y), len(table(bits)) // 2, 0)).astype(np.uint8)


def quantise(x, bits):
    """x [rows, K] of float32 values (in any float type) -> codes [rows, Kp], one a byte, scale bytes [rows, Kp / 32]"""
    x = np.asarray(x, np.float64)
    rows, K = x.shape
    Kp = -(-K // 128) * 128
    p = np.zeros((rows, Kp))
    p[:, :K] = x
    p = p.reshape(rows, Kp // 32, 32)
    fin = np.isfinite(p)
    byte = scale_bytes(np.abs(np.where(fin, p, 0)).max(-1), bits)
    codes = nearest(np.where(fin, p, 0) * 2.0 ** (127.0 - byte[..., None]), bits)
    if bits == 8:
        codes[~fin] = 0x7F
    else:
        bad = ~fin.all(-1)
        codes[bad], byte[bad] = 0, 255
    return codes.reshape(rows, Kp), byte.astype(np.uint8)


def values(codes, scales, bits):
    """[rows, Kp] of codes (one a byte) and [rows, Kp / 32] of scale bytes -> what they stand for"""
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return table(bits)[codes] * np.repeat(s, 32, axis=-1)


def pair(codes):
    return codes[..., 0::2] | codes[..., 1::2] << 4


def unpair(b):
    return np.stack((b & 15, b >> 4), -1).reshape(*b.shape[:-1], -1)


def pack_weights(codes, scales, N, K):
    """the packed buffer of include/sjd.h, byte by byte"""
    nt, kg = -(-N // 16), -(-K // 512)
    out = np.zeros((nt, kg, 4352), np.uint8)
    n, k = np.meshgrid(np.arange(N), np.arange(0, codes.shape[1], 2), indexing="ij")
    t, f, g, s, q, j = n // 16, n % 16, k // 512, k % 512 // 128, k % 128 // 32, k % 32 // 2
    out[t, g, 1024 * s + 16 * (16 * q + f) + j] = pair(codes)
    n, b = np.meshgrid(np.arange(N), np.arange(scales.shape[1]), indexing="ij")
    out[n // 16, b // 16, 4096 + 4 * (16 * (b % 4) + n % 16) + b % 16 // 4] = scales
    return out.reshape(-1)


# ---- the 8-bit cache ----
def cache_at(hd):
    """byte of K[p][d] and of V[p][d] in a block's record"""
    p, d = np.meshgrid(np.arange(32), np.arange(hd), indexing="ij")
    o, l = p // 16 * (hd // 32) + d // 32, 16 * (d % 32 // 8) + p % 16
    k = 1024 * (o // 2) + 16 * l + 8 * (o % 2) + d % 8
    o, l = d // 16, 16 * (p % 16 // 4) + d % 16
    return k, 32 * hd + 1024 * (o // 2) + 16 * l + 8 * (o % 2) + 4 * (p // 16) + p % 4


class Cache:
    def __init__(self, n_seqs, n_kv, hd, cap, fill=0xAB):
        self.hd, self.cap, self.at = hd, cap, cache_at(hd)
        self.codes = np.full((n_seqs, n_kv, -(-cap // 32), 64 * hd), fill, np.uint8)
        self.scales = np.full((n_seqs, n_kv, -(-cap // 32), 2), fill, np.uint8)

    def append(self, k, v, length, L):
        """k, v: [n_seqs, L, n_kv, hd]"""
        for b, n in enumerate(length):
            if n < 0 or n + L > self.cap:
                continue
            for h in range(self.codes.shape[1]):
                for blk in range(n // 32, (n + L - 1) // 32 + 1):
                    for i, x in enumerate((k, v)):
                        rec, p0 = self.codes[b, h, blk], 32 * blk
                        new = np.zeros((32, self.hd))
                        if p0 < n:
                            old = table(8)[rec[self.at[i]]] * 2.0 ** (float(self.scales[b, h, blk, i]) - 127)
                            new[: n - p0] = old[: n - p0]
                        lo, hi = max(n, p0), min(n + L, p0 + 32)
                        new[lo - p0:hi - p0] = x[b, lo - n:hi - n, h]
                        fin = np.isfinite(new)
                        byte = scale_byte(np.abs(np.where(fin, new, 0)).max(), 8)
                        c = nearest(np.where(fin, new, 0) * 2.0 ** (127.0 - byte), 8)
                        c[~fin] = 0x7F
                        rec[self.at[i]], self.scales[b, h, blk, i] = c, byte

    def values(self, b, h, n):
        """keys and values of the first n positions: [n, hd] each"""
        blocks = -(-n // 32)
        out = []
        for i in range(2):
            s = 2.0 ** (self.scales[b, h, :blocks, i].astype(np.float64) - 127)
            out.append((table(8)[self.codes[b, h, :blocks][:, self.at[i]]] * s[:, None, None]).reshape(-1, self.hd)[:n])
        return out


def attention(cache, q, length, L, n_heads, window, sinks):
    """q [n_seqs, L, n_heads, hd] -> (out, bound of sum |q k| / sqrt(hd) over visible keys, largest visible |v|), NaN rows for sequences that sit out"""
    n_seqs, n_kv, hd = cache.codes.shape[0], cache.codes.shape[1], cache.hd
    out, mag, top = (np.full((n_seqs, L, n_heads, w), np.nan) for w in (hd, 1, 1))
    for b, n in enumerate(length):
        if n < 0 or n + L > cache.cap:
            continue
        pos, key = n + np.arange(L)[:, None], np.arange(n + L)[None]
        see = (key <= pos) & ((key > pos - window) | (key < sinks) if window else True)
        for h in range(n_heads):
            k, v = cache.values(b, h // (n_heads // n_kv), n + L)
            for i in range(L):
                kk, vv = k[see[i]], v[see[i]]
                s = kk @ q[b, i, h] / math.sqrt(hd)
                p = np.exp(s - s.max())
                out[b, i, h] = p @ vv / p.sum()
                mag[b, i, h] = (np.abs(kk) @ np.abs(q[b, i, h])).max() / math.sqrt(hd)
                top[b, i, h] = np.abs(vv).max()
    return out, mag, top
