"""Calls of the attention operators at the edges of their contract: the header's bounds on what a call writes, lengths
beyond a page table, positions far out, long runs of one workgroup, and what the decode form's probabilities may lose.

Bounds are those of test_gpu_attention.py, except where a test states its own.
"""
import numpy as np
import pytest

from oracle import attention as oa
from test_gpu_attention import U16, U32, Setup, _dev, _host, _stream, torch  # noqa: F401 (torch: the fixture)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------- probabilities' bits

@pytest.mark.parametrize("heads,kv_heads,d,page,nq", [(8, 1, 128, 64, 1), (32, 4, 128, 16, 1), (3, 3, 64, 32, 5),
                                                      (24, 1, 128, 32, 1), (8, 1, 64, 64, 4)])
@pytest.mark.parametrize("kv", [[90, 33, 2], [2000, 700, 1300]])
def test_few_rows_keep_sixteen_bits_of_a_probability(torch, heads, kv_heads, d, page, nq, kv):
    """Up to 32 rows of a key/value head: a probability is two bf16 terms, off by 2^-8 of what the first leaves of it, so by
    2^-16; the sum it is divided by is fp32's own.  The output's rounding is then all that bf16 costs."""
    s = Setup([nq] * 3, kv, heads, kv_heads, d, page, "bf16", seed=21)
    got = _host(s.run()).astype(np.float64)
    want, spread, reach = oa.attend(s.cache, _host(s.q), s.q_start, s.kv, s.pages, True, s.scale, np.full(got.shape, 7.0))
    n = max(s.kv)
    rel = 2 * (d + 4) * U32 * reach[..., None] + 8 * U32 + 2 * (n / 4 + 32) * U32 + 2.0 ** -16
    bound = rel * spread + U16 * np.abs(want) * (1 + rel) + (6 * n + 1) * 2.0 ** -126
    off = np.abs(got - want)
    assert np.all(off <= bound), np.max(off / bound)
