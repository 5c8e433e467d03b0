"""CPU tests of the bound that the experts' precision is held to: what it takes as enough, and what it does not."""
import numpy as np
import pytest

from oracle import experts as ox

MAGNITUDE = ox.MAGNITUDE


def bf16(v):
    """v in bf16, to the nearest, ties to even."""
    w = np.asarray(v, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return ((w + 0x7fff + ((w >> 16) & 1)) & 0xffff0000).astype(np.uint32).view(np.float32).astype(np.float64)


def terms(v):
    """v as two bf16 terms, the first one cut off."""
    high = (np.asarray(v, dtype=np.float32).view(np.uint32) & 0xffff0000).view(np.float32).astype(np.float64)
    return high + bf16(v - high)


@pytest.mark.parametrize("keep_h,keep_y,within", [(np.float32, np.float32, True), (terms, np.float32, True), (bf16, np.float32, False),
                                                  (terms, bf16, False)])
def test_the_bound_sees_a_rounding_to_bf16(keep_h, keep_y, within):
    rng = np.random.default_rng(7)
    T, n, K, D, I = 40, 6, 3, 128, 96

    def few_bits(*shape):
        return MAGNITUDE[rng.integers(0, 8, size=shape)] * rng.choice([-1.0, 1.0], size=shape)

    x, gu, dn = few_bits(T, D), few_bits(n, 2 * I, D) / 32, few_bits(n, D, I) / 32
    topk, gates = rng.integers(0, n, size=(T, K)), rng.random((T, K)).astype(np.float32).astype(np.float64)
    kept = dict(u_h=2.0 ** -16, u_y=0.0, sums=False)
    res = bf16(-ox.experts(x, gu, dn, topk, gates, None, False, **kept)[0])
    want, bound = ox.experts(x, gu, dn, topk, gates, res, False, **kept)
    out = res.copy()
    for t in range(T):
        for k in range(K):
            g, u = np.split(gu[topk[t, k]] @ x[t], 2)
            h = np.asarray(keep_h((g / (1 + np.exp(-g)) * u)), dtype=np.float64)
            out[t] += gates[t, k] * np.asarray(keep_y(dn[topk[t, k]] @ h), dtype=np.float64)
    assert np.all(np.abs(out - want) <= bound) == within
    if not within:
        assert (np.abs(out - want) > bound).mean() > 0.1
