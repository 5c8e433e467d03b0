"""CPU tests of the 4-bit matrices and the expert routing: the plain forms on hand-worked values, the entry points' refusals."""
import os

import numpy as np
import pytest

from oracle import attention as oa
from oracle import experts as ox
from paper_2607_24787_amd import spp

# the addresses below are none: a call that is not refused must find no device
no_gpu = pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="refusals are checked where there is no GPU")

GOOD = 1 << 24


def test_quantise_is_the_caches():
    rng = np.random.default_rng(0)
    x = (rng.normal(size=(60, 96)) * np.exp(rng.uniform(-40, 40, size=(60, 1)))).astype(np.float32)
    x[0, :8] = [7.0, -6.0, 5.0, 0.25, 0.75, -1.25, 3.5, 2.5]
    x[1, 32:36] = [7.0000005, 0.5, -1.5, -0.0]
    x[2, 0], x[3, 40], x[4, 64:] = np.inf, np.nan, 0.0
    x[5, 3], x[6, 5] = np.finfo(np.float32).max, 1e-45
    for e in range(-126, 127, 9):   # largest magnitudes at the border of two scales
        x[7 + e % 50, 0] = 7.0 * 2.0 ** min(e, 125)
    codes, scales = ox.quantise(x)
    want_codes, want_scales = oa.quantise(x)
    assert np.array_equal(scales, want_scales) and np.array_equal(codes, want_codes)
    ok = ~np.isnan(oa.values(codes, scales))
    assert np.array_equal(ox.values(codes, scales)[ok], oa.values(codes, scales)[ok])
    assert np.array_equal(ox.unpack(ox.pack(codes)), codes)


def test_bound_of_quantised_covers_its_inputs():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(40, 64))
    err = np.abs(rng.normal(size=x.shape)) * 0.02
    q, bound = ox.quantised(x, err)
    for _ in range(50):
        other = ox.values(*ox.quantise(x + err * rng.uniform(-1, 1, size=x.shape)))
        assert np.all(np.abs(other - q) <= bound)
    assert np.all(ox.quantised(x, 0 * err)[1] == 0)


def test_sort_hand_worked():
    start, pair, place = ox.sort([[2, 0], [0, 7], [2, -1]], 3)
    assert start.tolist() == [0, 2, 2, 4]
    assert pair.tolist() == [1, 2, 0, 4, -1, -1]
    assert place.tolist() == [2, 0, 1, -1, 3, -1]


def test_experts_hand_worked():
    # one expert of one unit-like row: G = U = D = ones on the first element
    gu, dn = np.zeros((1, 64, 32)), np.zeros((1, 32, 32))
    gu[0, 0, 0], gu[0, 32, 0], dn[0, 5, 0] = 1.0, 2.0, 4.0
    x = np.zeros((1, 32))
    x[0, 0] = 3.0
    out, bound = ox.experts(x, gu, dn, np.array([[0]]), np.array([[0.5]]), None, False)
    want = 3.0 / (1 + np.exp(-3.0)) * 6.0 * 4.0 * 0.5
    assert abs(out[0, 5] - want) < 1e-12 and np.count_nonzero(out) == 1
    assert 0 < bound[0, 5] < 0.02 * want


# ------------------------------------------------------------------ refusals

def _refused(call, *args):
    with pytest.raises(spp.SppError) as e:
        call(*args)
    assert e.value.status == spp.SPP_EINVAL and str(e.value).strip()


def _not_refused(call, *args):
    with pytest.raises(spp.SppError) as e:    # what is left is that there is no device
        call(*args)
    assert e.value.status == spp.SPP_EHIP


def mx4(rows=6, cols=64, codes=GOOD, scales=3 * GOOD + 1):
    return spp.make_mx4(codes, scales, rows, cols)


BAD_MATRICES = [dict(cols=0), dict(cols=16), dict(cols=48), dict(cols=-32), dict(cols=(1 << 17) + 32), dict(rows=-1),
                dict(rows=1 << 31), dict(rows=1 << 30, cols=2048), dict(codes=0), dict(scales=0), dict(codes=GOOD + 8)]

QUANT = dict(dtype=1, x_dev=5 * GOOD, x_stride=64, q=mx4())
LOAD = dict(q=mx4(), dtype=1, out_dev=5 * GOOD, out_stride=64)
MATMUL = dict(w=mx4(rows=30), groups=3, start_dev=7 * GOOD, x_dev=5 * GOOD, x_stride=64, M=9, dtype=1, out_dev=6 * GOOD,
              out_stride=10)
MATMUL4 = dict(w=mx4(rows=30), groups=3, start_dev=7 * GOOD, x=mx4(rows=9, codes=5 * GOOD, scales=8 * GOOD), M=9, dtype=1,
               out_dev=6 * GOOD, out_stride=10)
EXPERTS = dict(gate_up=mx4(rows=5 * 2 * 32, cols=64), down=mx4(rows=5 * 64, cols=32, codes=2 * GOOD, scales=4 * GOOD), n=5,
               act=0, x_dev=5 * GOOD, x_stride=64, topk_dev=6 * GOOD, gates_dev=7 * GOOD, T=3, K=2, residual_dev=8 * GOOD,
               residual_stride=64, out_dev=9 * GOOD, out_stride=64, workspace_dev=10 * GOOD, workspace_bytes=1 << 40)
SORT = dict(topk_dev=GOOD, T=40, K=4, n=8, start_dev=2 * GOOD, pair_dev=3 * GOOD, place_dev=4 * GOOD, workspace_dev=0,
            workspace_bytes=0)
GATHER = dict(dtype=1, x_dev=GOOD, x_stride=64, place_dev=2 * GOOD, T=5, K=2, D=64, rows_dev=3 * GOOD, rows_stride=64)
COMBINE = dict(dtype=1, rows_dev=GOOD, rows_stride=64, place_dev=2 * GOOD, weights_dev=3 * GOOD, T=5, K=2, D=64,
               residual_dev=4 * GOOD, residual_stride=64, out_dev=5 * GOOD, out_stride=64)
GRAD = dict(dtype=1, d_out_dev=GOOD, d_out_stride=64, rows_dev=2 * GOOD, rows_stride=64, place_dev=3 * GOOD,
            weights_dev=4 * GOOD, T=5, K=2, D=64, d_rows_dev=5 * GOOD, d_rows_stride=64, d_weights_dev=6 * GOOD)

REFUSED = (
    [(spp.spp_mx4_quantize, QUANT, dict(q=mx4(**m))) for m in BAD_MATRICES]
    + [(spp.spp_mx4_load, LOAD, dict(q=mx4(**m))) for m in BAD_MATRICES]
    + [(spp.spp_mx4_matmul, MATMUL, dict(w=mx4(**{"rows": 30, **m}))) for m in BAD_MATRICES]
    + [(spp.spp_mx4_matmul_mx4, MATMUL4, dict(x=mx4(**{"rows": 9, "codes": 5 * GOOD, "scales": 8 * GOOD, **m}))) for m in BAD_MATRICES]
    + [(spp.spp_mx4_experts, EXPERTS, dict(gate_up=mx4(**{"rows": 320, **m}))) for m in BAD_MATRICES]
    + [(spp.spp_mx4_experts, EXPERTS, dict(down=mx4(**{"rows": 320, "cols": 32, "codes": 2 * GOOD, **m}))) for m in BAD_MATRICES]
    + [(spp.spp_mx4_quantize, QUANT, c) for c in (
        dict(dtype=2), dict(dtype=-1), dict(x_dev=0), dict(x_dev=5 * GOOD + 8), dict(x_stride=63), dict(x_stride=68),
        dict(x_stride=-64), dict(x_stride=1 << 31), dict(x_dev=GOOD), dict(x_dev=3 * GOOD), dict(q=mx4(scales=GOOD + 100)))]
    + [(spp.spp_mx4_load, LOAD, c) for c in (
        dict(dtype=3), dict(out_dev=0), dict(out_dev=5 * GOOD + 2), dict(out_stride=32), dict(out_stride=65),
        dict(out_stride=1 << 40), dict(out_dev=GOOD + 16), dict(out_dev=3 * GOOD))]
    + [(spp.spp_mx4_matmul, MATMUL, c) for c in (
        dict(groups=0), dict(groups=-1), dict(groups=4), dict(groups=31), dict(groups=1025), dict(start_dev=0),
        dict(start_dev=7 * GOOD + 2), dict(M=-1), dict(M=(1 << 24) + 1), dict(dtype=2), dict(out_dev=0),
        dict(out_dev=6 * GOOD + 1), dict(out_stride=9), dict(out_stride=-10), dict(out_stride=1 << 31), dict(x_dev=0),
        dict(x_dev=5 * GOOD + 4), dict(x_stride=56), dict(x_stride=70), dict(x_stride=1 << 40), dict(out_dev=5 * GOOD),
        dict(out_dev=GOOD + 30 * 32 - 2), dict(out_dev=3 * GOOD + 2), dict(out_dev=7 * GOOD), dict(dtype=0, out_dev=6 * GOOD + 2),
        dict(w=mx4(rows=0)), dict(w=mx4(rows=1 << 16), groups=1, M=(1 << 20) + 1, out_stride=1 << 16), dict(w=mx4(rows=(1 << 20) + 1), groups=1, out_stride=1 << 21))]
    + [(spp.spp_mx4_matmul_mx4, MATMUL4, c) for c in (
        dict(groups=7), dict(M=8), dict(x=mx4(rows=9, cols=32)), dict(x=mx4(rows=10)), dict(dtype=2), dict(out_dev=0),
        dict(out_stride=9), dict(out_dev=5 * GOOD + 16), dict(out_dev=8 * GOOD))]
    + [(spp.spp_mx4_experts, EXPERTS, c) for c in (
        dict(n=0), dict(n=4), dict(n=1025), dict(act=2), dict(act=-1), dict(T=-1), dict(T=1 << 24), dict(K=0), dict(K=65),
        dict(x_dev=0), dict(x_dev=5 * GOOD + 8), dict(x_stride=32), dict(x_stride=68), dict(topk_dev=0),
        dict(topk_dev=6 * GOOD + 1), dict(gates_dev=0), dict(gates_dev=7 * GOOD + 2), dict(residual_dev=8 * GOOD + 4),
        dict(residual_stride=60), dict(out_dev=0), dict(out_dev=9 * GOOD + 2), dict(out_stride=33), dict(out_dev=5 * GOOD),
        dict(out_dev=6 * GOOD), dict(out_dev=7 * GOOD), dict(out_dev=GOOD), dict(out_dev=4 * GOOD),
        dict(out_dev=8 * GOOD + 64), dict(out_dev=8 * GOOD, out_stride=128), dict(workspace_dev=0),
        dict(workspace_dev=10 * GOOD + 8), dict(workspace_bytes=0))]
    + [(spp.spp_expert_sort, SORT, c) for c in (
        dict(T=-1), dict(K=0), dict(T=1 << 24), dict(n=0), dict(n=1025), dict(topk_dev=0), dict(start_dev=0), dict(pair_dev=0),
        dict(place_dev=0), dict(topk_dev=GOOD + 2), dict(pair_dev=3 * GOOD + 1), dict(place_dev=3 * GOOD + 4),
        dict(pair_dev=GOOD), dict(start_dev=4 * GOOD + 636), dict(place_dev=GOOD - 4), dict(T=5000), dict(T=5000, workspace_dev=8 * GOOD, workspace_bytes=16),
        dict(T=5000, workspace_dev=8 * GOOD + 4, workspace_bytes=1 << 20))]
    + [(spp.spp_expert_gather, GATHER, c) for c in (
        dict(dtype=2), dict(T=-1), dict(K=0), dict(D=0), dict(D=4), dict(D=(1 << 20) + 8), dict(x_dev=0), dict(x_dev=GOOD + 2),
        dict(x_stride=56), dict(x_stride=65), dict(place_dev=0), dict(place_dev=2 * GOOD + 2), dict(rows_dev=0),
        dict(rows_stride=60), dict(rows_dev=GOOD + 512), dict(rows_dev=GOOD - 16))]
    + [(spp.spp_expert_combine, COMBINE, c) for c in (
        dict(dtype=-1), dict(T=-5), dict(K=-1), dict(D=12), dict(rows_dev=0), dict(rows_stride=8), dict(place_dev=0),
        dict(weights_dev=3 * GOOD + 2), dict(residual_dev=4 * GOOD + 8), dict(residual_stride=9), dict(out_dev=0),
        dict(out_stride=63), dict(out_dev=GOOD), dict(out_dev=4 * GOOD + 128), dict(out_dev=4 * GOOD, out_stride=128))]
    + [(spp.spp_expert_combine_grad, GRAD, c) for c in (
        dict(dtype=5), dict(T=-1), dict(K=0), dict(D=20), dict(d_out_dev=0), dict(d_out_stride=63), dict(rows_dev=0),
        dict(rows_stride=7), dict(place_dev=0), dict(weights_dev=1), dict(d_rows_dev=5 * GOOD + 4), dict(d_rows_stride=32),
        dict(d_weights_dev=6 * GOOD + 2), dict(d_rows_dev=GOOD), dict(d_rows_dev=2 * GOOD + 128),
        dict(d_rows_dev=2 * GOOD, d_rows_stride=72), dict(d_weights_dev=5 * GOOD + 64))]
)


@no_gpu
@pytest.mark.parametrize("call,good,change", REFUSED,
                         ids=[f"{i}-{c.__name__}-{'-'.join(d)}" for i, (c, _, d) in enumerate(REFUSED)])
def test_refusals(call, good, change):
    _refused(lambda: call(**{**good, **change}))


@no_gpu
@pytest.mark.parametrize("call,good", [
    (spp.spp_mx4_quantize, QUANT), (spp.spp_mx4_load, LOAD), (spp.spp_mx4_matmul, MATMUL), (spp.spp_mx4_matmul_mx4, MATMUL4),
    (spp.spp_mx4_experts, EXPERTS), (spp.spp_expert_sort, SORT), (spp.spp_expert_gather, GATHER),
    (spp.spp_expert_combine, COMBINE), (spp.spp_expert_combine_grad, GRAD),
    (spp.spp_mx4_experts, {**EXPERTS, "out_dev": 8 * GOOD}), (spp.spp_mx4_experts, {**EXPERTS, "residual_dev": 0}),
    (spp.spp_expert_combine, {**COMBINE, "out_dev": 4 * GOOD}), (spp.spp_expert_combine, {**COMBINE, "weights_dev": 0}),
    (spp.spp_expert_combine_grad, {**GRAD, "d_rows_dev": 2 * GOOD}), (spp.spp_expert_combine_grad, {**GRAD, "d_rows_dev": 0}),
    (spp.spp_expert_combine_grad, {**GRAD, "d_weights_dev": 0, "rows_dev": 0}),
    (spp.spp_mx4_matmul, {**MATMUL, "groups": 1, "start_dev": 0, "out_stride": 30, "M": 1})])
def test_sound_calls_reach_the_device(call, good):
    _not_refused(lambda: call(**good))


@no_gpu
def test_null_matrices():
    L = spp.lib()
    assert L.spp_mx4_quantize(1, GOOD, 64, None, None) == spp.SPP_EINVAL
    assert L.spp_mx4_load(None, 1, GOOD, 64, None) == spp.SPP_EINVAL
    assert L.spp_mx4_matmul(None, 1, None, GOOD, 64, 1, 1, GOOD, 64, None) == spp.SPP_EINVAL


@no_gpu
def test_calls_with_nothing_to_do():
    spp.spp_mx4_quantize(1, 0, 64, mx4(rows=0, codes=0, scales=0))
    spp.spp_mx4_load(mx4(rows=0, codes=0, scales=0), 1, 0, 64)
    spp.spp_mx4_matmul(**{**MATMUL, "M": 0, "x_dev": 0, "out_dev": 0})
    spp.spp_mx4_matmul_mx4(**{**MATMUL4, "M": 0, "x": mx4(rows=0, codes=0, scales=0), "out_dev": 0})
    spp.spp_mx4_experts(**{**EXPERTS, "T": 0, "x_dev": 0, "topk_dev": 0, "gates_dev": 0, "out_dev": 0, "workspace_dev": 0})
    spp.spp_expert_gather(**{**GATHER, "T": 0, "x_dev": 0})
    spp.spp_expert_combine(**{**COMBINE, "T": 0, "rows_dev": 0})
    spp.spp_expert_combine_grad(**{**GRAD, "T": 0, "rows_dev": 0})
    spp.spp_expert_combine_grad(**{**GRAD, "d_rows_dev": 0, "d_weights_dev": 0})


def test_workspaces_never_shrink_with_more_tokens():
    for n, D, I, K in ((128, 2048, 768, 8), (1, 32, 32, 1), (64, 1280, 896, 6), (1024, 256, 64, 64)):
        sizes = [spp.spp_mx4_experts_workspace(n, D, I, T, K) for T in
                 (0, 1, 2, 3, 5, 8, 16, 31, 64, 100, 128, 200, 255, 256, 257, 300, 500, 512, 1000, 1024, 2000, 4096, 8191, 50000)]
        assert all(s > 0 for s in sizes) and sizes == sorted(sizes)
        sorts = [spp.spp_expert_sort_workspace(T, 1, n) for T in
                 (0, 1, 4096, 8191, 8192, 12287, 12288, 100000, 262143, 262144, 262145, 300000, 1 << 20, 1 << 24)]
        assert all(s > 0 for s in sorts) and sorts == sorted(sorts)
    for bad in ((0, 64, 64, 1, 1), (1025, 64, 64, 1, 1), (4, 48, 64, 1, 1), (4, 64, 40, 1, 1), (4, 64, 64, -1, 1), (4, 64, 64, 1, 0),
                (4, 64, 64, 1, 65), (4, 1 << 14, 64, (1 << 19) + 1, 8), (4, 64, 64, 1 << 20, 32)):
        _refused(spp.spp_mx4_experts_workspace, *bad)
    for bad in ((-1, 1, 4), (1, 0, 4), (1 << 24, 2, 4), (4, 4, 0), (4, 4, 1025)):
        _refused(spp.spp_expert_sort_workspace, *bad)


@no_gpu
def test_a_workspace_is_enough_for_every_smaller_call():
    """A call whose workspace is too small says so before it finds no device."""
    rng = np.random.default_rng(0)
    for _ in range(300):
        n, K = int(rng.integers(1, 200)), int(rng.integers(1, 9))
        D, I = 32 * int(rng.integers(1, 60)), 32 * int(rng.integers(1, 40))
        T = int(np.exp(rng.uniform(0, np.log(9000))))
        need = spp.spp_mx4_experts_workspace(n, D, I, T, K)
        less = max(1, int(T * rng.uniform(0, 1)))
        gu, dn = mx4(rows=n * 2 * I, cols=D, codes=1 << 40, scales=1 << 42), mx4(rows=n * D, cols=I, codes=1 << 41, scales=1 << 43)
        call = dict(gate_up=gu, down=dn, n=n, act=int(rng.integers(0, 2)), x_dev=1 << 44, x_stride=D, topk_dev=1 << 45, gates_dev=1 << 46,
                    T=less, K=K, residual_dev=0, residual_stride=0, out_dev=1 << 47, out_stride=D, workspace_dev=1 << 48)
        _not_refused(lambda: spp.spp_mx4_experts(**call, workspace_bytes=need))
        P = int(np.exp(rng.uniform(0, np.log(400000))))
        need, less = spp.spp_expert_sort_workspace(P, 1, n), max(1, int(P * rng.uniform(0.7, 1)))
        _not_refused(lambda: spp.spp_expert_sort(1 << 40, less, 1, n, 1 << 41, 1 << 42, 1 << 43, 1 << 44, need))
