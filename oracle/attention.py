"""Plain CPU forms of the attention operators (numpy; 64 bits, except where the operator's definition rounds to 32).

Shares no code with the device path.  Cache format: see include/spp.h.
"""
from __future__ import annotations

import numpy as np

MAGNITUDE = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
VALUE = np.concatenate([MAGNITUDE, -MAGNITUDE])


def rotary_table(pos, axis_of, inv_freq):
    """[T, 2, F] cos and sin (64 bits): pos int [axes, T], axis_of [F], inv_freq fp32 [F]."""
    angle = np.asarray(pos, dtype=np.float64)[np.asarray(axis_of)].T * np.asarray(inv_freq, dtype=np.float32).astype(np.float64)
    return np.stack([np.cos(angle), np.sin(angle)], axis=1)


def rotate(x, table):
    """x [T, H, d] (fp32 values) turned by table [T, 2, F] (fp32): every product and sum rounded to fp32."""
    x = np.asarray(x, dtype=np.float32)
    if table is None:
        return x
    F = table.shape[2]
    cos, sin = table[:, None, 0].astype(np.float32), table[:, None, 1].astype(np.float32)
    out = x.copy()
    a, b = x[..., :F], x[..., F:2 * F]
    out[..., :F] = a * cos - b * sin
    out[..., F:2 * F] = b * cos + a * sin
    return out


def quantise(x):
    """(codes uint8 [..., d], scale bytes uint8 [..., d/32]) of fp32 x, block by block."""
    x = np.asarray(x, dtype=np.float32)
    blocks = x.reshape(x.shape[:-1] + (-1, 32))
    codes = np.zeros(blocks.shape, dtype=np.uint8)
    scales = np.zeros(blocks.shape[:-1], dtype=np.uint8)
    for at in np.ndindex(scales.shape):
        b = blocks[at].astype(np.float64)
        if not np.all(np.isfinite(b)):
            scales[at] = 255
            continue
        top = np.max(np.abs(b))
        e = -125
        while e < 125 and top > 7.0 * 2.0 ** e:
            e += 1
        scales[at] = e + 127
        r = np.abs(b) / 2.0 ** e
        gap = np.abs(r[:, None] - MAGNITUDE[None, :])
        near = gap == gap.min(axis=1, keepdims=True)
        # a tie between two codes goes to the even one
        even_first = np.where(near, np.arange(8) % 2, 2)
        codes[at] = np.argmin(even_first, axis=1) + 8 * np.signbit(blocks[at])
    return codes.reshape(x.shape), scales


def values(codes, scales):
    """fp64 values of codes [..., d] with scale bytes [..., d/32]."""
    blocks = VALUE[codes].reshape(codes.shape[:-1] + (-1, 32))
    unit = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int32) - 127))
    return (blocks * unit[..., None]).reshape(codes.shape)


class Cache:
    """A cache's bytes [n_pages, n_kv_heads, page * (d + d/16)], read and written one token's head at a time."""

    def __init__(self, n_kv_heads, d, page, n_pages, raw=None):
        self.h, self.d, self.page, self.n = n_kv_heads, d, page, n_pages
        shape = (n_pages, n_kv_heads, page * (d + d // 16))
        self.raw = np.zeros(shape, dtype=np.uint8) if raw is None else np.array(raw, dtype=np.uint8).reshape(shape)

    def _places(self, kv, slot):
        p, off = divmod(int(slot), self.page)
        half, n = self.d // 2, self.page * self.d
        first = (kv * self.page + off) * half
        scales = n + kv * n // 32 + np.arange(self.d // 32) * self.page + off
        return p, slice(first, first + half), scales

    def write(self, kv, slot, codes, scales):
        """codes [H, d], scales [H, d/32] of one token."""
        if not 0 <= slot < self.n * self.page:
            return
        p, c, s = self._places(kv, slot)
        self.raw[p, :, c] = codes[:, 0::2] | (codes[:, 1::2] << 4)
        self.raw[p][:, s] = scales

    def codes(self, kv, slot):
        p, c, s = self._places(kv, slot)
        pair = self.raw[p, :, c]
        return np.stack([pair & 15, pair >> 4], axis=-1).reshape(self.h, self.d), self.raw[p][:, s]

    def read(self, kv, slot):
        """fp64 [H, d]."""
        return values(*self.codes(kv, slot))


def store(cache, q, k, v, table, slots):
    """Writes k, v [T, Hkv, d] and returns the rotated queries (fp32, before their rounding to the storage type)."""
    kc, ks = quantise(rotate(k, table))
    vc, vs = quantise(v)
    for t, slot in enumerate(slots):
        cache.write(0, slot, kc[t], ks[t])
        cache.write(1, slot, vc[t], vs[t])
    return None if q is None else rotate(q, table)


def attend(cache, q, q_start, kv_len, pages, causal, scale, out):
    """out [n_tokens, Hq, d] (its rows of no sequence stay).  Also returns, for error bounds, sum_t p_t |v_t| per element
    and max_t scale * sum |q| |k_t| per (token, head)."""
    q = np.asarray(q, dtype=np.float64)
    out = np.array(out, dtype=np.float64)
    spread, reach = np.zeros(out.shape), np.zeros(out.shape[:2])
    G = q.shape[1] // cache.h
    for b, n in enumerate(kv_len):
        whole = max(int(n), 0)
        n = min(whole, len(pages[b]) * cache.page)
        nq = q_start[b + 1] - q_start[b]
        k, v = np.full((n, cache.h, cache.d), np.nan), np.full((n, cache.h, cache.d), np.nan)
        for t in range(n):
            p = pages[b][t // cache.page]
            if 0 <= p < cache.n:
                slot = p * cache.page + t % cache.page
                k[t], v[t] = cache.read(0, slot), cache.read(1, slot)
        for j in range(nq):
            i = q_start[b] + j
            seen = whole - nq + j + 1 if causal else whole
            out[i] = 0.0
            if seen <= 0:
                continue
            for h in range(q.shape[1]):
                kk, vv = k[:seen, h // G], v[:seen, h // G]
                z = scale * (kk @ q[i, h])
                with np.errstate(all="ignore"):
                    p = np.exp(z - np.max(z))
                    p = p / np.sum(p)
                    out[i, h] = np.nan if whole > n else p @ vv
                    spread[i, h] = p @ np.abs(vv)
                    reach[i, h] = scale * np.max(np.abs(kk) @ np.abs(q[i, h]))
    return out, spread, reach
