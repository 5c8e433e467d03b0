"""What the experts' FFN keeps between its steps: 16 bits of a SwiGLU result (SPP_ACT_BF16), fp32 of an expert's result.

The output's rounding, half a step of bf16, hides what a step before it loses, so
the residual here is minus the sum in bf16: what is left is at most 2^-8 of it and
its rounding 2^-16.  The first product's sums are exact in fp32: x and the weights
are small multiples of one half, times a power of two.  What the bound then holds:
the SwiGLU in fp32, its result's half a step of 16 bits (2^-16; in 4 bits, what an
input so close to a border may change), the second product's fp32 sums (I + 32 of
2 u32), the gates' sum.
"""
import numpy as np
import pytest

from oracle import experts as ox
from tests.test_gpu_experts import Experts, ids
from tests.test_gpu_mx4 import U, blank, dev, host, torch  # noqa: F401

pytestmark = pytest.mark.gpu

U_TERMS = 2.0 ** -16


def few_bits(rng, shape):
    """Multiples of one half up to 6, which 4 bits hold with the scale 1."""
    v = ox.MAGNITUDE[rng.integers(0, 8, size=shape)] * rng.choice([-1.0, 1.0], size=shape)
    v[..., ::32] = 6.0
    return v


def exact_experts(T, n, K, D, I, kind, seed):
    e = Experts(T, n, K, D, I, kind, seed=seed)
    rng = np.random.default_rng(seed + 1)
    for m, cols in ((e.gu, D), (e.dn, I)):
        m.codes, m.scales = ox.quantise(few_bits(rng, m.codes.shape))
        m.scales = m.scales - 2 - int(np.log2(cols) / 2)      # sums of the order of 1
        m.upload()
    e.x[:, :D] = dev(few_bits(rng, (T, D)), "bf16")
    return e


def want_of(e, act, residual):
    return ox.experts(host(e.x[:, :e.D]), e.gu.v.reshape(e.n, 2 * e.I, e.D), e.dn.v.reshape(e.n, e.D, e.I), host(e.topk_dev),
                      host(e.gates), residual, act == "mx4", u_h=U_TERMS, u_y=0.0, sums=False)


def check_kept(e, act):
    e.res[:, :e.D] = dev(-want_of(e, act, None)[0], "bf16")
    want, bound = want_of(e, act, host(e.res[:, :e.D]))
    bound = bound + U["bf16"] * (np.abs(want) + bound)
    got = host(e.run(act))[:e.T, :e.D]
    worst = np.max(np.abs(got - want) / np.maximum(bound, 1e-300))
    assert worst <= 1, worst


FEW = [(1, 16, 8, 128, 64, "distinct"), (1, 8, 3, 256, 32, "distinct"), (2, 40, 8, 96, 160, "bad"), (3, 8, 2, 64, 96, "any"),
       (20, 24, 5, 128, 64, "bad"), (70, 40, 4, 160, 224, "distinct")]
TILES = [(400, 8, 3, 128, 160, "bad"), (1300, 8, 4, 64, 288, "distinct"), (900, 64, 6, 96, 64, "any"), (3000, 3, 2, 64, 96, "any")]


@pytest.mark.parametrize("T,n,K,D,I,kind", FEW + TILES)
def test_results_of_4_bit_products_stay_in_fp32(torch, T, n, K, D, I, kind):  # noqa: F811
    check_kept(exact_experts(T, n, K, D, I, kind, T + I), "mx4")


@pytest.mark.parametrize("T,n,K,D,I,kind", FEW + TILES)
def test_swiglu_results_keep_16_bits(torch, T, n, K, D, I, kind):  # noqa: F811
    check_kept(exact_experts(T, n, K, D, I, kind, T + I), "bf16")


@pytest.mark.parametrize("T,n,K", [(1, 4, 2), (2, 8, 3), (5, 8, 2), (40, 4, 3), (300, 4, 2)])
@pytest.mark.parametrize("u_exp,finite", [(64, True), (66, False), (-60, True)])
def test_swiglu_results_at_the_largest_floats(torch, T, n, K, u_exp, finite):  # noqa: F811
    """h = 1.99994 * 2^127 is finite in fp32 and would round to infinity in bf16; 4 h is infinite, and so is its output."""
    D, I = 96, 64
    e = Experts(T, n, K, D, I, "distinct", residual=False)
    gu, dn = np.zeros((n, 2 * I, D)), np.zeros((n, D, I))
    gu[:, 0, :2] = 1.0                                   # g = x0 + x1
    gu[:, I, 2] = 1.0                                    # u = x2
    dn[:, :, 0] = 1.5
    for m, v in ((e.gu, gu), (e.dn, dn)):
        m.codes, m.scales = ox.quantise(v.reshape(m.codes.shape))
        m.upload()
        assert np.array_equal(m.v, v.reshape(m.codes.shape))
    e.dn.scales = e.dn.scales - 60
    e.dn.upload()
    x = np.zeros((T, D))
    x[:, :3] = [255 / 128 * 2.0 ** 63, 127 / 128 * 2.0 ** 56, 2.0 ** u_exp]
    e.x[:, :D] = dev(x, "bf16")
    assert np.array_equal(host(e.x[:, :D]), x)
    got = host(e.run("bf16"))[:T, :D]
    h = (x[:, 0] + x[:, 1]) * x[:, 2]
    want = h * 1.5 * 2.0 ** -60 * host(e.gates).sum(1)
    if finite:      # h's 16 bits, sums of K fp32 gates, the output's rounding
        assert np.all(np.abs(got - want[:, None]) <= (U_TERMS + (K + 3) * 2 * ox.U32 + U["bf16"]) * want[:, None] * (1 + 1e-3))
    else:
        assert np.isposinf(got).all()
