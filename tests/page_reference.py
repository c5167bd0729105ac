"""Rotary positions, the paged cache, its attention and the norms between blocks from their definitions, in 64 bits (numpy)."""
from __future__ import annotations

import math

import numpy as np


def frequencies(rot, theta=10000.0, scaling=0, factor=1.0, original=0.0, slow=1.0, fast=32.0):
    if scaling == 2:
        theta = theta * factor ** (rot / (rot - 2))
    f = np.array([theta ** (-2 * i / rot) for i in range(rot // 2)])
    if scaling == 1:
        f = f / factor
    if scaling == 3:
        w = np.clip((original * f / (2 * math.pi) - slow) / (fast - slow), 0, 1)
        f = w * f + (1 - w) * f / factor
    return f


def turns(f):
    return np.array([round(x / (2 * math.pi) * 2 ** 64) % 2 ** 64 for x in f], dtype=np.uint64).view(np.int64)


def rotate(x, pos, table, interleaved=False, magnitude=1.0, inverse=False):
    """x [rows, n, hd]; table: int64 turns.  Angles are exact modulo whole turns."""
    rot = 2 * len(table)
    angle = np.array([[int(p) * int(np.uint64(t)) % 2 ** 64 / 2 ** 64 * 2 * math.pi for t in table.view(np.uint64)] for p in pos])
    c, s = np.cos(angle)[:, None] * magnitude, np.sin(angle)[:, None] * magnitude * (-1 if inverse else 1)
    y = np.array(x, dtype=np.float64)
    one, two = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = y[..., one].copy(), y[..., two].copy()
    y[..., one], y[..., two] = a * c - b * s, b * c + a * s
    return y


def record_at(hd, bf16):
    """places of K[p][d] and V[p][d] in a record: two arrays [32, hd]"""
    E = 8 if bf16 else 4
    k, v = np.zeros((32, hd), np.int64), np.zeros((32, hd), np.int64)
    for p in range(32):
        t, j, h, i = p // 16, p // 8 % 2, p // 4 % 2, p % 4
        u, e = (2 * t + h, 4 * j + i) if bf16 else (p // 4, p % 4)
        for d in range(hd):
            k[p, d] = E * (32 * (d // E) + p) + d % E
            v[p, d] = 32 * hd + E * (1024 // E * (d // 32) + 32 * u + d % 32) + e
    return k, v


def fits(n, m, width, page):
    return n >= 0 and n + m <= width * page


def store(cache, rows_k, rows_v, start, length, table, page, bf16):
    """keys and values [rows, kv, hd] into cache [pages, kv, page / 32, 64 hd], in place"""
    n_pages, kv, _, rec = cache.shape
    ak, av = record_at(rec // 64, bf16)
    for b in range(len(length)):
        m = start[b + 1] - start[b]
        if not fits(length[b], m, table.shape[1], page):
            continue
        for i in range(m):
            p = length[b] + i
            g = table[b, p // page]
            if 0 <= g < n_pages:
                cache[g][:, p % page // 32, ak[p % 32]] = rows_k[start[b] + i]
                cache[g][:, p % page // 32, av[p % 32]] = rows_v[start[b] + i]


def sequence(cache, row, page, n, bf16):
    """keys and values [n, kv, hd] of a table row's first n positions, and which of them are in the pool"""
    n_pages, kv, _, rec = cache.shape
    ak, av = record_at(rec // 64, bf16)
    k, v, held = np.zeros((n, kv, rec // 64)), np.zeros((n, kv, rec // 64)), np.zeros(n, bool)
    for p in range(n):
        g = row[p // page]
        if 0 <= g < n_pages:
            held[p] = True
            k[p], v[p] = cache[g][:, p % page // 32, ak[p % 32]], cache[g][:, p % page // 32, av[p % 32]]
    return k, v, held


def attention(cache, q, start, length, table, page, scale, bf16, window=0, sinks=0):
    """q [rows, heads, hd] -> (out, sum |q k| scale at its largest, the largest |v|, positions) of every row and head; rows outside all sequences NaN"""
    rows, heads, hd = q.shape
    out, mag, top = (np.full(s, np.nan) for s in ((rows, heads, hd), (rows, heads), (rows, heads)))
    for b in range(len(length)):
        m, n = start[b + 1] - start[b], length[b]
        if not fits(n, m, table.shape[1], page) or m == 0:
            continue
        k, v, held = sequence(cache, table[b], page, n + m, bf16)
        g, r = heads // k.shape[1], slice(start[b], start[b + 1])
        j, p = np.arange(n + m)[None], np.arange(n, n + m)[:, None]
        see = held[None] & (j <= p) & ((j > p - window) | (j < sinks) if window else True)
        some = see.any(-1)
        for h in range(heads):
            ks, vs = k[:, h // g], v[:, h // g]
            s = np.where(see, q[r, h] @ ks.T * scale, -np.inf)
            w = np.exp(s - np.where(some, s.max(-1), 0)[:, None])
            out[r, h] = np.where(some[:, None], w @ vs / np.maximum(w.sum(-1), 1e-300)[:, None], 0)
            mag[r, h] = np.where(see, np.abs(q[r, h]) @ np.abs(ks).T, 0).max(-1) * scale
            top[r, h] = np.where(see, np.abs(vs).max(-1)[None], 0).max(-1)
    return out, mag, top


def norm(x, resid, eps, post=None, gate=None, scale=1.0, pre=None):
    """(h, out) and the part that was added to resid"""
    y = x if post is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * post
    y = scale * (y if gate is None else gate * y)
    h = resid + y
    return h, None if pre is None else h / np.sqrt((h * h).mean(-1, keepdims=True) + eps) * pre, y
