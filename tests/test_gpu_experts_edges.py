"""The experts' operators at the ends of their ranges, on the device."""
import numpy as np
import pytest

from tests.test_gpu_experts import Experts, Sorted, ids
from tests.test_gpu_mx4 import Matrix, blank, dev, host, stream, torch  # noqa: F401

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


@pytest.mark.parametrize("M", [1, 9, 300])
def test_inputs_and_outputs_as_columns_of_one_buffer(torch, M):  # noqa: F811
    """The bits of calls with buffers of their own, and nothing else of the buffer changed."""
    from paper_2607_24787_amd import spp
    rng = np.random.default_rng(M)
    D, W, n, bf16 = 64, 200, 5, spp.DTYPE_BF16
    w, start = Matrix(rng, n * 40, D), dev(np.sort(np.r_[0, rng.integers(0, M + 1, n - 1), M]).astype(np.int32))
    e = Experts(M, n, 1, D, 32, pad=0, residual=False)
    s = Sorted(ids(rng, M, 1, n, "any"), n)
    gates = dev(rng.random(M).astype(np.float32))
    x = dev(rng.normal(size=(M, D)), "bf16")
    calls = {
        "matmul": (40, lambda x, xs, y, ys: spp.spp_mx4_matmul(w.desc, n, start.data_ptr(), x, xs, M, bf16, y, ys, stream())),
        "experts": (D, lambda x, xs, y, ys: spp.spp_mx4_experts(
            e.gu.desc, e.dn.desc, n, spp.ACT_MX4, x, xs, e.topk_dev.data_ptr(), e.gates.data_ptr(), M, 1, 0, 0, y, ys,
            e.space.data_ptr(), e.size, stream())),
        "gather": (D, lambda x, xs, y, ys: spp.spp_expert_gather(bf16, x, xs, s.place.data_ptr(), M, 1, D, y, ys, stream())),
        "combine": (D, lambda x, xs, y, ys: spp.spp_expert_combine(bf16, x, xs, s.place.data_ptr(), gates.data_ptr(), M, 1, D, 0, 0,
                                                                   y, ys, stream())),
        "gradient": (D, lambda x, xs, y, ys: spp.spp_expert_combine_grad(bf16, x, xs, 0, 0, s.place.data_ptr(), gates.data_ptr(), M,
                                                                         1, D, y, ys, 0, stream()))}
    for name, (N, call) in calls.items():
        alone, both = blank((M, N), "bf16"), blank((M + 1, W), "bf16")
        call(x.data_ptr(), D, alone.data_ptr(), N)
        both[:M, 72:72 + D] = x
        call(both.data_ptr() + 2 * 72, W, both.data_ptr() + 2 * 8, W)
        got = host(both)
        assert np.array_equal(got[:M, 8:8 + N], host(alone)), name
        assert np.array_equal(got[:M, 72:72 + D], host(x)), name
        got[:M, 8:8 + N] = got[:M, 72:72 + D] = np.nan
        assert np.isnan(got).all(), name


@pytest.mark.parametrize("T,K,D", [(3, 2, 8), (400, 3, 2048), (2000, 2, 4104)])
def test_rows_that_two_pairs_name(torch, T, K, D):  # noqa: F811
    """Each 16 bytes are one of the pairs'; rows that one pair names are its own, the others as they were."""
    from paper_2607_24787_amd import spp
    rng = np.random.default_rng(T)
    P = T * K
    place = rng.integers(0, P, size=P)
    x, place_dev = dev(rng.normal(size=(T, D)), "bf16"), dev(place.astype(np.int32))
    rows, d_rows = blank((P, D), "bf16"), blank((P, D), "bf16")
    spp.spp_expert_gather(spp.DTYPE_BF16, x.data_ptr(), D, place_dev.data_ptr(), T, K, D, rows.data_ptr(), D, stream())
    spp.spp_expert_combine_grad(spp.DTYPE_BF16, x.data_ptr(), D, 0, 0, place_dev.data_ptr(), 0, T, K, D, d_rows.data_ptr(), D, 0,
                                stream())
    sent = host(x).reshape(T, D // 8, 8)
    for got in (host(rows).reshape(P, D // 8, 8), host(d_rows).reshape(P, D // 8, 8)):
        fine = np.zeros((P, D // 8), dtype=bool)
        for p in range(P):
            fine[place[p]] |= (got[place[p]] == sent[p // K]).all(-1)
        named = np.isin(np.arange(P), place)
        assert fine[named].all() and np.isnan(got[~named]).all() and 0 < named.sum() < P


@pytest.mark.parametrize("M", [1, 20, 700])
def test_products_of_subnormal_activations(torch, M):  # noqa: F811
    """A bf16 below 2^-126 times a weight of 6 * 2^125 is a number like any other."""
    from oracle import experts as ox
    from paper_2607_24787_amd import spp
    rng = np.random.default_rng(M)
    N, K = 300, 96
    codes, scales = rng.integers(0, 16, size=(N, K)).astype(np.uint8), np.full((N, K // 32), 252, dtype=np.uint8)
    x = dev(rng.integers(-127, 128, size=(M, K)) * 2.0 ** -133, "bf16")
    b, s, out = dev(ox.pack(codes)), dev(scales), blank((M, N), "f32")
    spp.spp_mx4_matmul(spp.make_mx4(b.data_ptr(), s.data_ptr(), N, K), 1, 0, x.data_ptr(), K, M, spp.DTYPE_F32, out.data_ptr(), N,
                       stream())
    v = x.view(torch.int16).cpu().numpy().astype(np.int64)
    exact = np.where(v < 0, -1.0, 1.0) * (v & 0x7fff) * 2.0 ** -133
    assert np.abs(exact).max() < 2.0 ** -126 and np.abs(exact).max() > 0
    want, bound = ox.product(exact, ox.values(codes, scales))
    assert np.all(np.abs(host(out) - want) <= bound + ox.U32 * np.abs(want))
