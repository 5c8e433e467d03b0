"""Plain CPU forms of the 4-bit matrices' and the expert routing's operators (numpy, 64 bits).

Shares no code with the device path.  Format and contracts: see include/spp.h.
Errors: where a function takes or gives `err`, it is a bound on how far the
device's value may be from the exact one, element by element.
"""
from __future__ import annotations

import numpy as np

MAGNITUDE = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BORDER = (MAGNITUDE[1:] + MAGNITUDE[:-1]) / 2
U16, U32 = 2.0 ** -8, 2.0 ** -24


def scale_bytes(top):
    """The scale byte of blocks whose largest magnitude is top."""
    top = np.asarray(top, dtype=np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.ceil(np.log2(top / 7.0))
    e = np.where(np.isfinite(e), e, -125)
    e = np.where(top > 7.0 * np.exp2(e), e + 1, np.where(top <= 7.0 * np.exp2(e - 1), e - 1, e))
    byte = np.clip(e, -125, 125).astype(np.int64) + 127
    return np.where(np.isfinite(top), byte, 255)


def to_codes(x, byte):
    """Codes of x [..., 32] with scale bytes [..., 1]: the nearest magnitude, a tie to the even code."""
    r = np.abs(x) / np.exp2(byte - 127.0)
    code = np.zeros(x.shape, dtype=np.int64)
    for j, border in enumerate(BORDER):
        code += (r > border) | ((r == border) & (j % 2 == 1))
    return code + 8 * np.signbit(x)


def quantise(x):
    """(codes uint8 [..., C], scale bytes uint8 [..., C/32])."""
    blocks = np.asarray(x, dtype=np.float64).reshape(x.shape[:-1] + (-1, 32))
    finite = np.isfinite(blocks).all(-1, keepdims=True)
    top = np.where(finite, np.abs(blocks).max(-1, keepdims=True), np.inf)
    byte = scale_bytes(top)
    codes = np.where(finite, to_codes(np.where(finite, blocks, 0.0), np.where(finite, byte, 127)), 0)
    return codes.reshape(x.shape).astype(np.uint8), byte[..., 0].astype(np.uint8)


def values(codes, scales):
    """fp64 values of codes [..., C] with scale bytes [..., C/32]."""
    v = np.concatenate([MAGNITUDE, -MAGNITUDE])[codes].reshape(codes.shape[:-1] + (-1, 32))
    unit = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (v * unit[..., None]).reshape(codes.shape)


def pack(codes):
    """Codes [..., C] as bytes [..., C/2], the even element low."""
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def unpack(b):
    return np.stack([b & 15, b >> 4], axis=-1).reshape(b.shape[:-1] + (-1,))


def quantised(x, err):
    """(values in 4 bits of x [..., C], bound): the bound holds for every input within err of x."""
    q = values(*quantise(x))
    low, high = np.abs(x) - err, np.abs(x) + err

    def top(a):
        return scale_bytes(np.maximum(a, 0.0).reshape(a.shape[:-1] + (-1, 32)).max(-1, keepdims=True))

    worst = np.zeros(x.shape)
    for byte in (top(low), top(high)):
        for end in (x - err, x + err):
            blocks = end.reshape(end.shape[:-1] + (-1, 32))
            code = to_codes(blocks, byte)
            v = np.concatenate([MAGNITUDE, -MAGNITUDE])[code] * np.exp2(byte - 127.0)
            worst = np.maximum(worst, np.abs(v.reshape(x.shape) - q))
    return q, worst


def product(x, w, err=None):
    """(x w^T, bound): fp32 sums of exact products; x within err.  An addition is off by at most 2 u32 of what it adds up
    to (it may cut off instead of rounding), K products and 32 parts."""
    reach = np.abs(x) @ np.abs(w).T
    bound = (x.shape[-1] + 32) * 2 * U32 * reach + 2.0 ** -126 * (x.shape[-1] + 1)
    if err is not None:
        bound = bound + err @ np.abs(w).T * (1 + 1e-3)
    return x @ w.T, bound


def groups_of(start, M):
    """Rows of each group."""
    at = np.clip(np.asarray(start), 0, M)
    return [np.arange(a, b) for a, b in zip(at[:-1], at[1:])]


def experts(x, gate_up, down, topk, gates, residual, mx4, u_h=U16, u_y=U16, sums=True):
    """(out, bound) of the routed experts before the output's rounding.

    x [T, D]; gate_up [n, 2I, D], down [n, D, I] values; topk, gates [T, K]; residual [T, D] or None.
    u_h: half a step, relative, of what holds the SwiGLU's result (with mx4: 4 bits); u_y: of each expert's result.
    sums=False: the first product's sums are exact in fp32, as the inputs see to.
    """
    T, D = x.shape
    n, I = gate_up.shape[0], gate_up.shape[1] // 2
    err_x = np.zeros(x.shape)
    if mx4:
        x, err_x = quantised(x, err_x)
    out = np.zeros((T, D)) if residual is None else residual.copy()
    reach = np.abs(out)
    bound = np.zeros((T, D))
    for e in range(n):
        t, k = np.nonzero(topk == e)
        if t.size == 0:
            continue
        gu, err = product(x[t], gate_up[e])
        err = err if sums else 0 * err
        g, u = gu[:, :I], gu[:, I:]
        s = g / (1 + np.exp(-g))
        h = s * u
        # |silu'| is at most 1.1; the fp32 function itself 16 u32 of its value, its argument's exponential |g| u32 more
        err_h = 1.1 * err[:, :I] * (np.abs(u) + err[:, I:]) + np.abs(s) * err[:, I:] + (16 + np.abs(g)) * U32 * np.abs(h) + 2.0 ** -126
        if mx4:
            h, err_h = quantised(h, err_h)
        else:
            err_h = err_h + u_h * (np.abs(h) + err_h)
        y, err_y = product(h, down[e], err_h)
        err_y = err_y + u_y * (np.abs(y) + err_y)
        w = gates[t, k][:, None]
        np.add.at(out, t, w * y)
        np.add.at(reach, t, np.abs(w) * (np.abs(y) + err_y))
        np.add.at(bound, t, np.abs(w) * err_y)
    return out, bound + (topk.shape[1] + 2) * 2 * U32 * reach


def sort(topk, n):
    """(start [n+1], pair [P], place [P])."""
    ids = np.asarray(topk).reshape(-1)
    ok = (ids >= 0) & (ids < n)
    order = [p for e in range(n) for p in np.nonzero(ids == e)[0]]
    pair = np.full(ids.size, -1, dtype=np.int64)
    place = np.full(ids.size, -1, dtype=np.int64)
    pair[:len(order)] = order
    place[order] = np.arange(len(order))
    count = np.bincount(ids[ok], minlength=n)
    return np.concatenate([[0], np.cumsum(count)]), pair, place
