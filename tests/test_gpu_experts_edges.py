"""The experts' operators at the ends of their ranges, on the device."""
import numpy as np
import pytest

from tests.test_gpu_mx4 import blank, dev, host, stream, torch  # noqa: F401

pytestmark = pytest.mark.gpu


def test_gather_and_combine_of_the_most_tokens(torch):  # noqa: F811
    """2^24 tokens with rows that take a whole workgroup each at fewer tokens: 2^32 threads, more than a launch has."""
    from paper_2607_24787_amd import spp
    T, D = 1 << 24, 1032
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("70 GB")
    x, rows = (torch.empty((T + 1, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    place = torch.arange(T - 1, -1, -1, dtype=torch.int32, device="cuda")
    seen = torch.tensor([0, 1, 2, 3, 255, T // 2 - 1, T // 2, T // 2 + 1, T - 257, T - 2, T - 1], device="cuda")
    x[seen] = dev(np.random.default_rng(0).normal(size=(len(seen), D)), "bf16")
    rows[T] = 3.0
    w = torch.full((T,), 0.5, device="cuda")
    spp.spp_expert_gather(spp.DTYPE_BF16, x.data_ptr(), D, place.data_ptr(), T, 1, D, rows.data_ptr(), D, stream())
    assert torch.equal(rows[T - 1 - seen], x[seen])
    # and back: x's own rows halved, from their places
    sent = x[seen].clone()
    x[T] = 3.0
    spp.spp_expert_combine(spp.DTYPE_BF16, rows.data_ptr(), D, place.data_ptr(), w.data_ptr(), T, 1, D, 0, 0, x.data_ptr(), D,
                           stream())
    assert torch.equal(x[seen], sent / 2)
    assert (x[T] == 3.0).all() and (rows[T] == 3.0).all()
    del x, rows
    torch.cuda.empty_cache()
