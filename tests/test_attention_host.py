"""CPU tests of the attention operators: the plain forms on hand-worked values, the entry points' refusals, the axes helper."""
import os

import numpy as np
import pytest

from oracle import attention as oa
from paper_2607_24787_amd import spp

# the addresses below are none: a call that is not refused must find no device
pytestmark = pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="refusals are checked where there is no GPU")

GOOD = 1 << 20   # a 16-byte aligned address: refused calls never read it


def test_quantise_hand_worked():
    x = np.zeros((1, 64), dtype=np.float32)
    x[0, :8] = [7.0, -6.0, 5.0, 0.25, 0.75, -1.25, 3.5, 2.5]      # scale 1: 7 -> 6 (half a step), ties to the even code
    x[0, 32:36] = [7.0000005, 0.5, -1.5, -0.0]                    # past 7: scale 2
    codes, scales = oa.quantise(x)
    assert scales.tolist() == [[127, 128]]
    assert codes[0, :9].tolist() == [7, 15, 6, 0, 2, 10, 6, 4, 0]
    assert codes[0, 32:37].tolist() == [6, 0, 10, 8, 0]
    v = oa.values(codes, scales)
    assert v[0, :8].tolist() == [6.0, -6.0, 4.0, 0.0, 1.0, -1.0, 4.0, 2.0]
    assert v[0, 32:36].tolist() == [8.0, 0.0, -2.0, 0.0]


def test_quantise_extremes():
    x = np.zeros((5, 32), dtype=np.float32)
    x[1, 3] = np.inf
    x[2, 0], x[2, 1] = np.nan, 1.0
    x[3, 5] = np.finfo(np.float32).max
    x[4, 6] = 1e-45
    codes, scales = oa.quantise(x)
    assert scales[:, 0].tolist() == [2, 255, 255, 252, 2]
    assert codes[3, 5] == 7 and np.isfinite(np.float32(oa.values(codes, scales)[3, 5]))
    assert codes[4].max() == 0


def test_no_element_is_off_by_more_than_half_its_step():
    rng = np.random.default_rng(0)
    x = (rng.normal(size=(200, 128)) * np.exp(rng.uniform(-20, 20, size=(200, 1)))).astype(np.float32)
    codes, scales = oa.quantise(x)
    unit = np.repeat(np.ldexp(1.0, scales.astype(int) - 127), 32, axis=-1)
    a = np.abs(x.astype(np.float64)) / unit
    assert a.max() <= 7.0
    step = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))
    assert np.all(np.abs(oa.values(codes, scales) - x) <= step * unit / 2)
    # and the scale is the smallest that allows it
    top = a.reshape(200, 4, 32).max(-1)
    assert np.all(top > 3.5)


def test_cache_places_do_not_overlap():
    c = oa.Cache(2, 64, 16, 2)
    for slot in range(32):
        for kv in range(2):
            q = np.full((2, 64), 1 + kv, dtype=np.uint8)
            c.write(kv, slot, q, np.full((2, 2), 100 + slot, dtype=np.uint8))
    for slot in range(32):
        for kv in range(2):
            q, s = c.codes(kv, slot)
            assert np.all(q == 1 + kv) and np.all(s == 100 + slot)
    assert np.all(c.raw > 0)   # every byte belongs to something


def test_plain_attention_rows_that_see_nothing_and_prefixes():
    c = oa.Cache(1, 64, 16, 1)
    rng = np.random.default_rng(1)
    k, v = rng.normal(size=(2, 3, 1, 64))
    oa.store(c, None, k, v, None, [0, 1, 2])
    q = rng.normal(size=(5, 1, 64))
    out, _, _ = oa.attend(c, q, [0, 5], [3], [[0]], True, 0.1, np.ones((5, 1, 64)))
    assert np.all(out[:2] == 0)                       # five queries, three tokens: the first two see none
    assert np.allclose(out[2, 0], c.read(1, 0)[0])    # one token: its value


def test_rotary_axes():
    assert spp.rotary_axes([4, 2, 2], False).tolist() == [0, 0, 0, 0, 1, 1, 2, 2]
    assert spp.rotary_axes([4, 2, 2], True).tolist() == [0, 1, 2, 0, 1, 2, 0, 0]
    assert spp.rotary_axes([8], True).tolist() == [0] * 8
    with pytest.raises(ValueError):
        spp.rotary_axes([5, 5, 0], True)
    with pytest.raises(ValueError):
        spp.rotary_axes([4, -1], False)


def test_cache_bytes():
    assert spp.spp_kv4_cache_bytes(spp.make_attn_desc(32, 4, 128, 64, 10)) == 10 * 4 * 64 * 136
    assert spp.spp_kv4_cache_bytes(spp.make_attn_desc(1, 1, 64, 16, 1)) == 16 * 68
    assert spp.spp_kv4_cache_bytes(spp.make_attn_desc(8, 8, 128, 256, 1 << 20)) == (1 << 20) * 8 * 256 * 136


BAD_DESCS = [(3, 2, 128, 64, 1), (0, 1, 128, 64, 1), (4, 0, 128, 64, 1), (2048, 1, 128, 64, 1), (4, 4, 96, 64, 1),
             (4, 4, 256, 64, 1), (4, 4, 128, 8, 1), (4, 4, 128, 48, 1), (4, 4, 128, 512, 1), (4, 4, 128, 64, 0),
             (4, 4, 128, 64, -1)]


def _refused(call, *args):
    with pytest.raises(spp.SppError) as e:
        call(*args)
    assert e.value.status == spp.SPP_EINVAL and str(e.value).strip()


@pytest.mark.parametrize("shape", BAD_DESCS)
def test_bad_shapes_are_refused(shape):
    d = spp.make_attn_desc(*shape)
    _refused(spp.spp_kv4_cache_bytes, d)
    _refused(spp.spp_kv4_attend_workspace, d, 1, 1, 1)
    _refused(spp.spp_kv4_store, d, GOOD, 1, 0, 0, 0, 0, GOOD, 1 << 20, GOOD, 1 << 20, 0, 0, GOOD, 1)
    _refused(spp.spp_kv4_load, d, GOOD, 1, GOOD, 1, GOOD, 1 << 20, 0, 0)
    _refused(spp.spp_kv4_attend, d, GOOD, 1, GOOD, 1 << 20, 0, GOOD, GOOD, 1, 1, 1, 1, 1, True, 1.0, GOOD * 64, 1 << 20,
             GOOD, 1 << 30)
    L = spp.lib()
    assert L.spp_kv4_cache_bytes(None) == 0
    assert L.spp_kv4_store(None, GOOD, 1, None, 0, None, 0, GOOD, 512, GOOD, 512, None, 0, GOOD, 1, None) == spp.SPP_EINVAL


DESC = spp.make_attn_desc(8, 2, 64, 16, 4)
TABLE = dict(pos_dev=GOOD, pos_stride=5, n_axes=3, axis_of=[0] * 8, inv_freq_dev=GOOD, T=5, table_dev=GOOD)
STORE = dict(desc=DESC, cache_dev=GOOD, dtype=1, q_dev=GOOD, q_stride=512, q_out_dev=GOOD * 2, q_out_stride=512,
             k_dev=GOOD, k_stride=128, v_dev=GOOD, v_stride=128, table_dev=GOOD, n_freq=32, slots_dev=GOOD, T=3)
LOAD = dict(desc=DESC, cache_dev=GOOD, dtype=1, slots_dev=GOOD, T=3, k_out_dev=GOOD, k_stride=128, v_out_dev=GOOD,
            v_stride=128)
ATTEND = dict(desc=DESC, cache_dev=GOOD, dtype=1, q_dev=GOOD, q_stride=512, q_start_dev=GOOD, kv_len_dev=GOOD,
              pages_dev=GOOD, pages_stride=4, n_seq=2, n_tokens=6, max_q=4, max_kv=64, causal=True, scale=0.125,
              out_dev=GOOD * 2, out_stride=512, workspace_dev=GOOD * 4, workspace_bytes=1 << 40)

REFUSED = (
    [(spp.spp_rotary_table, TABLE, c) for c in (
        dict(n_axes=0), dict(n_axes=5), dict(axis_of=[0] * 7), dict(axis_of=[0] * 12), dict(axis_of=[0] * 72),
        dict(axis_of=[]), dict(axis_of=[3] + [0] * 7), dict(axis_of=[-1] + [0] * 7), dict(T=-1), dict(T=1 << 30),
        dict(pos_dev=0), dict(pos_dev=GOOD + 2), dict(inv_freq_dev=0), dict(inv_freq_dev=GOOD + 1), dict(table_dev=0), dict(table_dev=GOOD + 4), dict(pos_stride=4),
        dict(pos_stride=-5), dict(pos_stride=1 << 60))]
    + [(spp.spp_kv4_store, STORE, c) for c in (
        dict(cache_dev=0), dict(cache_dev=GOOD + 8), dict(dtype=2), dict(dtype=-1), dict(q_dev=0), dict(q_out_dev=0),
        dict(q_dev=GOOD + 8), dict(q_stride=511), dict(q_stride=504), dict(q_stride=-512), dict(q_stride=1 << 62),
        dict(k_dev=0), dict(v_dev=0), dict(k_dev=GOOD + 2), dict(k_stride=120), dict(v_stride=132), dict(table_dev=0),
        dict(table_dev=GOOD + 4), dict(n_freq=0), dict(n_freq=12), dict(n_freq=40), dict(n_freq=-8), dict(slots_dev=0), dict(slots_dev=GOOD + 4),
        dict(T=-1), dict(T=1 << 30), dict(T=(1 << 27) // 12 + 1), dict(q_out_dev=GOOD + 16), dict(q_out_dev=GOOD + 1024),
        dict(q_out_dev=GOOD, q_out_stride=1024))]
    + [(spp.spp_kv4_load, LOAD, c) for c in (
        dict(cache_dev=0), dict(cache_dev=GOOD + 1), dict(dtype=7), dict(slots_dev=0), dict(T=-2), dict(T=1 << 30), dict(T=(1 << 25) + 1),
        dict(k_out_dev=GOOD + 4), dict(k_stride=64), dict(v_stride=129))]
    + [(spp.spp_kv4_attend, ATTEND, c) for c in (
        dict(cache_dev=0), dict(cache_dev=GOOD + 4), dict(dtype=3), dict(q_dev=0), dict(q_dev=GOOD + 6), dict(q_stride=500),
        dict(q_start_dev=0), dict(kv_len_dev=0), dict(pages_dev=0), dict(pages_stride=0), dict(pages_stride=-1),
        dict(pages_stride=1 << 27), dict(pages_stride=1 << 62), dict(n_seq=-1), dict(n_tokens=-1), dict(n_tokens=1 << 30), dict(max_q=0),
        dict(max_kv=-1), dict(max_q=1 << 29), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
        dict(scale=float("inf")), dict(scale=1e-60), dict(scale=3e38),
        dict(n_seq=1 << 24, n_tokens=1 << 24, max_q=1), dict(causal=2), dict(out_dev=0), dict(out_dev=GOOD + 512), dict(out_stride=1024, out_dev=GOOD),
        dict(workspace_dev=0), dict(workspace_dev=GOOD * 4 + 8), dict(workspace_bytes=0, max_kv=4096), dict(workspace_bytes=16384, max_kv=4096),
        dict(kv_len_dev=GOOD + 2), dict(pages_dev=GOOD + 1), dict(q_start_dev=GOOD + 2))]
)


@pytest.mark.parametrize("call,good,change", REFUSED, ids=[f"{c.__name__}-{'-'.join(f'{k}={v}' for k, v in d.items())}"[:60] for c, _, d in REFUSED])
def test_refusals(call, good, change):
    _refused(lambda: call(**{**good, **change}))


def test_strides_that_would_wrap_are_refused():
    for change in (dict(q_stride=(1 << 63) - 512), dict(k_stride=1 << 61), dict(q_stride=-(1 << 62))):
        _refused(lambda: spp.spp_kv4_store(**{**STORE, **change}))
    _refused(lambda: spp.spp_rotary_table(**{**TABLE, "pos_stride": (1 << 63) - 1}))


def test_calls_with_nothing_to_do():
    spp.spp_rotary_table(**{**TABLE, "T": 0})
    spp.spp_kv4_store(**{**STORE, "T": 0})
    spp.spp_kv4_load(**{**LOAD, "T": 0})
    spp.spp_kv4_load(**{**LOAD, "k_out_dev": 0, "v_out_dev": 0})
    spp.spp_kv4_attend(**{**ATTEND, "n_seq": 0, "n_tokens": 0})
    spp.spp_kv4_attend(**{**ATTEND, "n_tokens": 0})


def test_workspace_grows_with_the_work_and_needs_no_device():
    sizes = [1, 2, 3, 7, 16, 17, 64, 300, 5000]
    for heads, kv_heads, dim in ((32, 4, 128), (8, 8, 64), (16, 1, 128)):
        d = spp.make_attn_desc(heads, kv_heads, dim, 64, 100)
        for n in sizes:
            for q in sizes:
                for kv in (0, 200, 1000, 100000):
                    need = spp.spp_kv4_attend_workspace(d, n, q, kv)
                    assert 0 < need < (1 << 27)
                    # never less for more
                    assert need >= spp.spp_kv4_attend_workspace(d, max(1, n // 2), max(1, q // 3), kv // 2)


@pytest.mark.parametrize("dtype", [0, 1])
def test_a_workspace_is_enough_for_every_smaller_call(dtype):
    """A call whose workspace is too small says so before anything else is found wrong with the device."""
    rng = np.random.default_rng(0)
    for _ in range(400):
        kv_heads = int(rng.integers(1, 9))
        d = spp.make_attn_desc(kv_heads * int(rng.integers(1, 9)), kv_heads, int(rng.choice([64, 128])), 16, 4)
        n, q, kv = (int(np.exp(rng.uniform(0, np.log(m)))) for m in (2000, 600, 200000))
        need = spp.spp_kv4_attend_workspace(d, n, q, kv)
        small = [max(1, int(v * f)) for v, f in zip((n, q, kv), rng.uniform(0, 1, size=3))]
        row = d.n_heads * d.head_dim
        with pytest.raises(spp.SppError) as e:
            spp.spp_kv4_attend(d, GOOD, dtype, GOOD, row, GOOD, GOOD, GOOD, 1, small[0], 1, small[1], small[2], True, 0.1,
                               GOOD * 64, row, GOOD * 4, need)
        assert "workspace" not in str(e.value), (d.n_heads, kv_heads, n, q, kv, small)


# ------------------------------------------------------- outputs that overlap rows

ROW, KV = 8 * 64 * 2, 2 * 64 * 2       # bytes of DESC's query rows, of its key or value rows (bf16)
WIDE = ROW + 2 * KV                    # one fused row: queries, keys, values


def _fused(**change):
    """A call on rows of one fused product, in elements."""
    return dict(STORE, q_dev=GOOD, q_stride=WIDE // 2, q_out_dev=GOOD, q_out_stride=WIDE // 2, k_dev=GOOD + ROW,
                k_stride=WIDE // 2, v_dev=GOOD + ROW + KV, v_stride=WIDE // 2, T=5, **change)


def _not_refused(call):
    with pytest.raises(spp.SppError) as e:    # what is left is that there is no device
        call()
    assert e.value.status == spp.SPP_EHIP


@pytest.mark.parametrize("change", [
    dict(k_dev=GOOD), dict(v_dev=GOOD + ROW - 16), dict(k_dev=GOOD + WIDE - 16), dict(v_dev=GOOD + 4 * WIDE),
    dict(k_dev=GOOD - WIDE + ROW - 16),
    # rotated queries beside the fused rows, keys where they go
    dict(q_out_dev=2 * GOOD, q_out_stride=ROW // 2, k_dev=2 * GOOD + 3 * ROW, k_stride=KV // 2),
    dict(q_out_dev=2 * GOOD, q_out_stride=ROW // 2, v_dev=2 * GOOD - 4 * WIDE - KV + 16),
    dict(q_out_dev=2 * GOOD, q_out_stride=2 * WIDE // 2, k_dev=2 * GOOD + WIDE, k_stride=WIDE // 2)])
def test_rotated_queries_over_keys_or_values_are_refused(change):
    _refused(lambda: spp.spp_kv4_store(**{**_fused(), **change}))


@pytest.mark.parametrize("change", [
    {}, dict(v_dev=GOOD + ROW), dict(k_dev=GOOD + 5 * WIDE), dict(k_dev=GOOD - 5 * WIDE + ROW),
    dict(q_out_dev=2 * GOOD, q_out_stride=ROW // 2, v_dev=2 * GOOD - 4 * WIDE - KV),
    # between the rows: at the same stride, and at twice the stride
    dict(q_dev=4 * GOOD, q_out_dev=2 * GOOD + WIDE, k_dev=2 * GOOD + ROW),
    dict(q_dev=4 * GOOD, q_out_dev=2 * GOOD, k_dev=2 * GOOD + ROW, k_stride=WIDE)])
def test_rotated_queries_beside_keys_and_values_are_taken(change):
    _not_refused(lambda: spp.spp_kv4_store(**{**_fused(), **change}))


def test_read_back_keys_over_values_are_refused():
    rows = dict(LOAD, T=4, k_stride=256, v_stride=256)
    for v in (GOOD, GOOD + 128, GOOD + 3 * 512, GOOD + 512 - 16, GOOD - 3 * 512 + 240):
        _refused(lambda: spp.spp_kv4_load(**{**rows, "v_out_dev": v}))
    for v in (GOOD + 256, GOOD - 256, GOOD + 4 * 512, GOOD - 3 * 512 - 256):
        _not_refused(lambda: spp.spp_kv4_load(**{**rows, "v_out_dev": v}))
