"""Float64 oracle of the paged low-bit cache and the attention over it (numpy, element by element; test infrastructure).

The head quantiser is Section 3's (Eq. 3 with b bits); position 0 of a sequence keeps 4 bits in a 3-bit cache.  Pages are
addressed as in a page table: position p of a sequence is slot p % page of page table[p // page].
"""
from __future__ import annotations

import math

import numpy as np


def quantise(x, bits, eps):
    """Head vectors (last axis) -> (integer codes, scale float64); x ~ scale * code."""
    x = np.asarray(x, np.float64)
    L = 2 ** (bits - 1) - 1
    gamma = np.abs(x).max(-1)
    s = L / (gamma + eps)
    q = np.clip(np.rint(s[..., None] * x), -(L + 1), L)
    return q.astype(np.int64), gamma / L


def rotate(x, pos, base):
    """RoPE of one head vector at one position: the pair (i, i + hd/2) turned by pos * base^(-2i/hd)."""
    x = np.asarray(x, np.float64)
    half = x.shape[-1] // 2
    out = np.empty_like(x)
    for i in range(half):
        angle = pos * float(base) ** (-2.0 * i / x.shape[-1])
        c, s = math.cos(angle), math.sin(angle)
        out[..., i] = x[..., i] * c - x[..., half + i] * s
        out[..., half + i] = x[..., half + i] * c + x[..., i] * s
    return out


def tokens(q_start, kv_len):
    """(row, sequence, index, position) of every new token."""
    for b in range(len(kv_len)):
        n = int(q_start[b + 1]) - int(q_start[b])
        for i in range(n):
            yield int(q_start[b]) + i, b, i, int(kv_len[b]) - n + i


def place(table, b, pos, page, n_pages):
    """(page, slot) of a position, or None without a page."""
    if pos < 0 or pos // page >= table.shape[1]:
        return None
    p = int(table[b, pos // page])
    return (p, pos % page) if 0 <= p < n_pages else None


class Cache:
    """Codes and scales of every slot, and 4-bit codes of position 0; unwritten slots hold zeros."""

    def __init__(self, bits, n_kv_heads, head_dim, page_size, n_pages):
        self.bits, self.heads, self.hd, self.page, self.n_pages = bits, n_kv_heads, head_dim, page_size, n_pages
        self.codes = np.zeros((2, n_pages, n_kv_heads, page_size, head_dim), np.int64)
        self.scales = np.zeros((2, n_pages, n_kv_heads, page_size))
        self.bos = np.zeros((2, n_pages, n_kv_heads, head_dim), np.int64)

    def write(self, q_start, kv_len, table, k, v, rope_base=0.0, eps=1e-5):
        k = np.asarray(k, np.float64).reshape(len(k), self.heads, self.hd)
        v = np.asarray(v, np.float64).reshape(len(v), self.heads, self.hd)
        for row, b, _, pos in tokens(q_start, kv_len):
            at = place(table, b, pos, self.page, self.n_pages)
            if at is None:
                continue
            for n, x in enumerate((rotate(k[row], pos, rope_base) if rope_base else k[row], v[row])):
                first = self.bits == 3 and pos == 0
                q, scale = quantise(x, 4 if first else self.bits, eps)
                if first:
                    self.bos[n, at[0]] = q
                else:
                    self.codes[n, at[0], :, at[1]] = q
                self.scales[n, at[0], :, at[1]] = scale

    def values(self, table, b, pos):
        """(key, value) heads of a position [heads, hd], or None."""
        at = place(table, b, pos, self.page, self.n_pages)
        if at is None:
            return None
        codes = self.bos[:, at[0]] if self.bits == 3 and pos == 0 else self.codes[:, at[0], :, at[1]]
        return codes * self.scales[:, at[0], :, at[1], None]

    def read(self, q_start, kv_len, table, n_tokens):
        out = np.zeros((2, n_tokens, self.heads, self.hd))
        for row, b, _, pos in tokens(q_start, kv_len):
            x = self.values(table, b, pos)
            if x is not None:
                out[:, row] = x
        return out

    def attend(self, q_start, kv_len, table, q, n_heads, scale=0.0, window=0, sinks=0):
        """(out, weighted absolute values, largest sum of absolute products of a seen score), [n_tokens, n_heads, hd],
        the same, and [n_tokens, n_heads]: the last two are what error bounds are made of."""
        q = np.asarray(q, np.float64).reshape(len(q), n_heads, self.hd)
        out, mag, top = np.zeros_like(q), np.zeros_like(q), np.zeros(q.shape[:2])
        scale = scale or 1.0 / math.sqrt(self.hd)
        group = n_heads // self.heads
        for b in range(len(kv_len)):
            reach = min(max(int(kv_len[b]), 0), table.shape[1] * self.page)
            held = [self.values(table, b, j) for j in range(reach)]
            there = np.array([x is not None for x in held], bool)
            zero = np.zeros((2, self.heads, self.hd))
            kv = np.stack([zero if x is None else x for x in held], 2) if reach else np.zeros((2, self.heads, 0, self.hd))
            j = np.arange(reach)
            for row, bb, _, pos in tokens(q_start, kv_len):
                if bb != b:
                    continue
                seen = there & (j <= pos)
                if window:
                    seen &= (j > pos - window) | (j < sinks)
                if not seen.any():
                    continue
                for h in range(n_heads):
                    K, V = kv[0, h // group][seen], kv[1, h // group][seen]
                    s = (K @ q[row, h]) * scale
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    out[row, h] = p @ V
                    mag[row, h] = p @ np.abs(V)
                    top[row, h] = (np.abs(K) @ np.abs(q[row, h])).max() * scale
        return out, mag, top


def unpack_pool(raw, bits, n_kv_heads, head_dim, page_size, n_pages):
    """Bytes of a pool -> (codes [2, pages, heads, page, hd], scales fp32 [2, pages, heads, page], bos codes [2, pages,
    heads, hd]); codes without their offset."""
    P = (head_dim + 31) // 32 * 32
    row = P * bits // 8
    chunk = 2 * page_size * row + 8 * page_size + (P if bits == 3 else 0)
    raw = np.asarray(raw, np.uint8)[:n_pages * n_kv_heads * chunk].reshape(n_pages, n_kv_heads, chunk)

    def entries(r, b):
        if b == 8:
            u = r.astype(np.int64)
        elif b == 4:
            u = np.stack((r & 15, r >> 4), -1).reshape(*r.shape[:-1], -1).astype(np.int64)
        else:
            w = np.ascontiguousarray(r).view("<u4").reshape(*r.shape[:-1], -1, 3).astype(np.int64)
            u = np.empty((*w.shape[:-1], 32), np.int64)
            for e in range(32):
                half, n = 16 * (e // 16), e % 16
                if n < 15:
                    u[..., e] = (w[..., n // 5] >> (half + 3 * (n % 5))) & 7
                else:
                    u[..., e] = sum(((w[..., t] >> (half + 15)) & 1) << t for t in range(3))
            u = u.reshape(*r.shape[:-1], -1)
        return u - 2 ** (b - 1)

    n = page_size * row
    codes = np.stack([entries(raw[:, :, i * n:(i + 1) * n].reshape(n_pages, n_kv_heads, page_size, row), bits) for i in (0, 1)])
    at = 2 * n
    scales = np.stack([np.ascontiguousarray(raw[:, :, at + 4 * i * page_size:at + 4 * (i + 1) * page_size]).view(np.float32) for i in (0, 1)])
    bos = None
    if bits == 3:
        at += 8 * page_size
        bos = np.stack([entries(raw[:, :, at + i * P // 2:at + (i + 1) * P // 2], 4) for i in (0, 1)])
    return codes, scales, bos
