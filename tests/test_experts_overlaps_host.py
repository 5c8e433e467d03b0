"""CPU tests of the overlaps that the 4-bit matrices' and the experts' calls refuse, against every byte of both sides.

The addresses are none: a call that is not refused must find no device.
"""
import numpy as np
import pytest

from paper_2607_24787_amd import spp
from tests.test_mx4_host import COMBINE, EXPERTS, GATHER, GOOD, GRAD, MATMUL, MATMUL4, _not_refused, _refused, mx4, no_gpu

pytestmark = no_gpu


def bytes_of(at, count, stride, row):
    """Addresses of `count` rows of `row` bytes, `stride` bytes apart."""
    return set((at + stride * np.arange(count)[:, None] + np.arange(row)).ravel().tolist())


def refused(call, **args):
    with pytest.raises(spp.SppError) as e:
        call(**args)
    assert e.value.status in (spp.SPP_EINVAL, spp.SPP_EHIP)
    return e.value.status == spp.SPP_EINVAL


def test_rows_that_share_a_byte_are_refused_and_no_others():
    rng = np.random.default_rng(0)
    seen = [0, 0]
    for _ in range(4000):
        T, K = (int(v) for v in rng.integers(1, 6, size=2))
        x_stride = 8 * int(rng.integers(1, 8))
        same = rng.random() < 0.5
        rows_stride = x_stride if same else 8 * int(rng.integers(1, 8))
        x_at, rows_at = (1 << 30) + 16 * int(rng.integers(0, 40)), (1 << 30) + 16 * int(rng.integers(0, 40))
        want = bool(bytes_of(x_at, T, 2 * x_stride, 16) & bytes_of(rows_at, T * K, 2 * rows_stride, 16))
        got = refused(spp.spp_expert_gather, **{**GATHER, "D": 8, "T": T, "K": K, "x_dev": x_at, "x_stride": x_stride,
                                                "rows_dev": rows_at, "rows_stride": rows_stride})
        assert got == want, (T, K, x_stride, rows_stride, x_at, rows_at)
        seen[want] += 1
    assert min(seen) > 400


def test_products_whose_rows_share_a_byte_are_refused_and_no_others():
    rng = np.random.default_rng(1)
    seen = [0, 0]
    for _ in range(4000):
        M, N = int(rng.integers(1, 6)), int(rng.integers(1, 30))
        x_stride = 32 + 8 * int(rng.integers(0, 6))
        out_stride = max(N, x_stride if rng.random() < 0.6 else int(rng.integers(1, 80)))
        x_at, out_at = (1 << 30) + 16 * int(rng.integers(0, 30)), (1 << 30) + 2 * int(rng.integers(0, 240))
        want = bool(bytes_of(x_at, M, 2 * x_stride, 64) & bytes_of(out_at, M, 2 * out_stride, 2 * N))
        got = refused(spp.spp_mx4_matmul, **{**MATMUL, "w": mx4(rows=N, cols=32), "groups": 1, "start_dev": 0, "x_dev": x_at,
                                             "x_stride": x_stride, "M": M, "out_dev": out_at, "out_stride": out_stride})
        assert got == want, (M, N, x_stride, out_stride, x_at, out_at)
        seen[want] += 1
    assert min(seen) > 400


# column ranges of one buffer of rows of 192: no byte is shared
@pytest.mark.parametrize("call,good,change", [
    (spp.spp_mx4_matmul, MATMUL, dict(x_stride=192, out_dev=5 * GOOD + 128, out_stride=192)),
    (spp.spp_mx4_matmul, MATMUL, dict(x_dev=5 * GOOD + 32, x_stride=192, out_dev=5 * GOOD, out_stride=192)),
    (spp.spp_mx4_experts, EXPERTS, dict(x_stride=192, out_dev=5 * GOOD + 128, out_stride=192)),
    (spp.spp_mx4_experts, EXPERTS, dict(residual_stride=192, out_dev=8 * GOOD + 256, out_stride=192)),
    (spp.spp_expert_gather, GATHER, dict(x_stride=192, rows_dev=GOOD + 128, rows_stride=192)),
    (spp.spp_expert_combine, COMBINE, dict(rows_stride=192, out_dev=GOOD + 128, out_stride=192)),
    (spp.spp_expert_combine, COMBINE, dict(residual_stride=192, out_dev=4 * GOOD + 128, out_stride=192)),
    (spp.spp_expert_combine_grad, GRAD, dict(d_out_stride=192, d_rows_dev=GOOD + 128, d_rows_stride=192)),
    (spp.spp_expert_combine_grad, GRAD, dict(rows_stride=192, d_rows_dev=2 * GOOD + 256, d_rows_stride=192))])
def test_column_ranges_of_one_buffer_are_accepted(call, good, change):
    _not_refused(lambda: call(**{**good, **change}))


OUTSIDE = 10 * GOOD    # where EXPERTS has its workspace
EXPERTS_T = {**EXPERTS, "T": 300, "residual_dev": 0, "workspace_bytes": 1 << 30}


@pytest.mark.parametrize("call,good,change", [
    (spp.spp_expert_gather, GATHER, dict(rows_dev=2 * GOOD)),
    (spp.spp_expert_gather, GATHER, dict(rows_dev=2 * GOOD + 32)),
    (spp.spp_expert_gather, GATHER, dict(place_dev=3 * GOOD + 10 * 128 - 4)),
    (spp.spp_expert_combine, COMBINE, dict(out_dev=2 * GOOD)),
    (spp.spp_expert_combine, COMBINE, dict(out_dev=3 * GOOD)),
    (spp.spp_expert_combine, COMBINE, dict(out_dev=3 * GOOD + 32)),
    (spp.spp_expert_combine, COMBINE, dict(place_dev=5 * GOOD + 5 * 128 - 4)),
    (spp.spp_expert_combine_grad, GRAD, dict(d_rows_dev=3 * GOOD)),
    (spp.spp_expert_combine_grad, GRAD, dict(d_rows_dev=4 * GOOD + 32)),
    (spp.spp_expert_combine_grad, GRAD, dict(d_rows_dev=4 * GOOD + 32, d_weights_dev=0)),
    (spp.spp_expert_combine_grad, GRAD, dict(d_weights_dev=GOOD + 636)),
    (spp.spp_expert_combine_grad, GRAD, dict(d_weights_dev=2 * GOOD)),
    (spp.spp_expert_combine_grad, GRAD, dict(d_weights_dev=3 * GOOD)),
    (spp.spp_expert_combine_grad, GRAD, dict(d_weights_dev=4 * GOOD)),
    (spp.spp_expert_combine_grad, GRAD, dict(d_weights_dev=4 * GOOD - 36, d_rows_dev=0)),
    (spp.spp_mx4_experts, EXPERTS, dict(workspace_dev=9 * GOOD)),
    (spp.spp_mx4_experts, EXPERTS, dict(workspace_dev=8 * GOOD + 256)),
    (spp.spp_mx4_experts, EXPERTS, dict(workspace_dev=7 * GOOD)),
    (spp.spp_mx4_experts, EXPERTS, dict(workspace_dev=6 * GOOD + 16)),
    (spp.spp_mx4_experts, EXPERTS, dict(workspace_dev=5 * GOOD)),
    (spp.spp_mx4_experts, EXPERTS, dict(workspace_dev=GOOD + 320 * 32 - 16)),
    (spp.spp_mx4_experts, EXPERTS, dict(workspace_dev=3 * GOOD)),
    (spp.spp_mx4_experts, EXPERTS, dict(workspace_dev=2 * GOOD)),
    (spp.spp_mx4_experts, EXPERTS, dict(workspace_dev=4 * GOOD + 304)),
    (spp.spp_mx4_experts, EXPERTS_T, dict(topk_dev=OUTSIDE + 4096)),
    (spp.spp_mx4_experts, EXPERTS_T, dict(out_dev=OUTSIDE - 16)),
] + [(spp.spp_expert_sort, {"topk_dev": GOOD, "T": 5000, "K": 4, "n": 8, "start_dev": 2 * GOOD, "pair_dev": 3 * GOOD,
                            "place_dev": 4 * GOOD, "workspace_dev": 5 * GOOD, "workspace_bytes": 1 << 20},
      dict(workspace_dev=at)) for at in (GOOD, 2 * GOOD + 32, 3 * GOOD + 79984, 4 * GOOD + 16)])
def test_outputs_and_workspaces_over_other_arrays_are_refused(call, good, change):
    _not_refused(lambda: call(**good))
    _refused(lambda: call(**{**good, **change}))


@pytest.mark.parametrize("call,good,change", [
    (spp.spp_expert_gather, GATHER, dict(rows_dev=2 * GOOD + 48)),
    (spp.spp_expert_combine, COMBINE, dict(out_dev=3 * GOOD + 48)),
    (spp.spp_expert_combine, COMBINE, dict(weights_dev=0, out_dev=3 * GOOD)),
    (spp.spp_expert_combine_grad, GRAD, dict(d_weights_dev=4 * GOOD + 40)),
    (spp.spp_expert_combine_grad, GRAD, dict(d_rows_dev=4 * GOOD - 1280)),
    (spp.spp_mx4_experts, EXPERTS, dict(workspace_dev=9 * GOOD + 384)),
    (spp.spp_expert_sort, {"topk_dev": GOOD, "T": 40, "K": 4, "n": 8, "start_dev": 2 * GOOD, "pair_dev": 3 * GOOD,
                           "place_dev": 4 * GOOD, "workspace_dev": GOOD, "workspace_bytes": 16}, dict())])
def test_neighbouring_arrays_are_accepted(call, good, change):
    _not_refused(lambda: call(**{**good, **change}))


def test_arrays_of_no_element_overlap_nothing():
    spp_sort = dict(topk_dev=GOOD + 4, T=0, K=4, n=8, start_dev=GOOD, pair_dev=GOOD + 8, place_dev=GOOD + 12, workspace_dev=0,
                    workspace_bytes=0)
    _not_refused(lambda: spp.spp_expert_sort(**spp_sort))
