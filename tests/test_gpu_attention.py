"""The attention operators on the device against their plain forms (oracle/attention.py).

Bounds.  u16 = 2^-8 is half a step of bf16 relative to the value, u32 = 2^-24 of
fp32.  Tables: 4 u32 (two units in the last place of the sine in [1/2, 1], the
correction and its rounding).  Stored codes and loaded values: equal.  Attention,
per element, with S = sum_t p_t |v_t| and reach = scale * max_t sum |q| |k_t|:
a score is a sum of d exact products in fp32 and is off by at most d u32 reach,
its power's argument by u32 reach more and the power by 2 u32, numerator and
denominator each: 2 (d + 4) u32 reach + 8 u32; the sums run over n tokens in
pieces of at least 4 per addition and a final tree, off by (n / 4 + 32) u32 each
(the running maximum's rescales are exact to 2 u32 a time and counted in it);
probabilities of bf16 queries are off by u16 each; the output by u16 or u32.
What is below the least normal number may become 0: a power below 2^-126 where
the largest is at least 1, so n times 2^-126 times the largest |v| (6 here, with
scales of at most 1), and the output itself: (6 n + 1) 2^-126 in all.
"""
import math

import numpy as np
import pytest

from oracle import attention as oa

pytestmark = pytest.mark.gpu

U16, U32 = 2.0 ** -8, 2.0 ** -24


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _code(dtype):
    from paper_2607_24787_amd import spp
    return spp.DTYPE_BF16 if dtype == "bf16" else spp.DTYPE_F32


def _stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def _dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def _host(t):
    return t.float().cpu().numpy()


class Setup:
    """A cache of random pages, sequences of given lengths, and their queries."""

    def __init__(self, nq, kv, heads, kv_heads, d, page, dtype, seed=0, spare=3, extra_rows=2):
        from paper_2607_24787_amd import spp
        rng = np.random.default_rng(seed)
        self.H, self.Hk, self.d, self.page, self.dtype = heads, kv_heads, d, page, dtype
        counts = [-(-k // page) for k in kv]
        self.n_pages = sum(counts) + spare
        self.desc = spp.make_attn_desc(heads, kv_heads, d, page, self.n_pages)
        order = rng.permutation(self.n_pages)
        self.wide = max(counts + [1]) + 1
        self.pages = np.full((len(kv), self.wide), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(counts):
            self.pages[b, :n] = order[at:at + n]
            at += n
        # codes of every value, scales of a normal cache; unused places hold garbage, NaN scales among it
        self.cache = oa.Cache(kv_heads, d, page, self.n_pages)
        self.cache.raw[:] = rng.integers(0, 256, size=self.cache.raw.shape, dtype=np.uint8)
        flat = self.cache.raw[:, :, page * d:]
        flat[:] = rng.integers(124, 128, size=flat.shape)
        used = np.zeros((self.n_pages, page), dtype=bool)
        for b, k in enumerate(kv):
            for t in range(k):
                used[self.pages[b, t // page], t % page] = True
        scales = self.cache.raw[:, :, page * d:].reshape(self.n_pages, kv_heads, 2, d // 32, page)
        junk = rng.integers(250, 256, size=scales.shape).astype(np.uint8)
        scales[:] = np.where(used[:, None, None, None], scales, junk)
        self.nq, self.kv = list(nq), list(kv)
        self.q_start = np.concatenate([[0], np.cumsum(nq)]).astype(np.int32)
        self.T = int(self.q_start[-1]) + extra_rows
        self.q = _dev(rng.normal(size=(self.T, heads, d)).astype(np.float32), dtype)
        self.scale = 1.0 / math.sqrt(d)

    def run(self, causal=True, max_q=None, max_kv=None, q=None, out=None, null_start=False, n_tokens=None, ws=None,
            kv_len=None, cache=None, q_stride=None, out_stride=None, wait=True):
        import torch
        from paper_2607_24787_amd import spp
        cache = _dev(self.cache.raw) if cache is None else cache
        max_q = max(self.nq + [1]) if max_q is None else max_q
        max_kv = max(self.kv) if max_kv is None else max_kv
        size = spp.spp_kv4_attend_workspace(self.desc, len(self.kv), max_q, max_kv)
        if ws is None:
            ws = torch.zeros(size + 64, dtype=torch.uint8, device="cuda")
            ws[size:] = 255
        q = self.q if q is None else q
        out = torch.full_like(q, 7.0) if out is None else out
        row = self.H * self.d
        keep = [_dev(self.q_start), _dev(np.asarray(self.kv if kv_len is None else kv_len, dtype=np.int32)), _dev(self.pages), cache]
        spp.spp_kv4_attend(self.desc, cache.data_ptr(), _code(self.dtype), q.data_ptr(), q_stride or row,
                           0 if null_start else keep[0].data_ptr(), keep[1].data_ptr(), keep[2].data_ptr(), self.wide,
                           len(self.kv), n_tokens or self.T, max_q, max_kv, causal, self.scale, out.data_ptr(),
                           out_stride or row, ws.data_ptr(), size, _stream())
        if wait:
            torch.cuda.synchronize()
            assert int(ws[-64:].min()) == 255    # nothing past the workspace
        return out

    def check(self, out, causal=True, kv_len=None, untouched=7.0):
        got = _host(out).astype(np.float64)
        want, spread, reach = oa.attend(self.cache, _host(self.q), self.q_start, self.kv if kv_len is None else kv_len, self.pages, causal, self.scale,
                                        np.full(got.shape, untouched))
        n = max(self.kv + [1])
        rel = 2 * (self.d + 4) * U32 * reach[..., None] + 8 * U32 + 2 * (n / 4 + 32) * U32
        rel = rel + (U16 if self.dtype == "bf16" else 0.0)
        bound = rel * spread + (U16 if self.dtype == "bf16" else U32) * np.abs(want) * (1 + rel) + (6 * n + 1) * 2.0 ** -126
        assert np.array_equal(np.isnan(got), np.isnan(want)), np.argwhere(np.isnan(got) != np.isnan(want))[:5]
        ok = np.isnan(want) | (np.abs(got - want) <= bound)
        assert ok.all(), (np.argwhere(~ok)[:5], got[~ok][:5], want[~ok][:5], np.broadcast_to(bound, got.shape)[~ok][:5])
        return want


# ------------------------------------------------------------------ rotary tables

@pytest.mark.parametrize("T,F,axes", [(1, 64, 3), (7, 8, 1), (33, 40, 4), (1000, 64, 3), (257, 16, 2)])
def test_rotary_table(torch, T, F, axes):
    from paper_2607_24787_amd import spp
    rng = np.random.default_rng(T)
    pos = rng.integers(-5, 1 << 24, size=(axes, T + 3)).astype(np.int32)
    pos[:, 0] = 0
    axis_of = rng.integers(0, axes, size=F).astype(np.int32)
    freq = (1e6 ** (-np.arange(F) / F)).astype(np.float32)
    table = torch.full((T + 1, 2, F), 9.0, device="cuda")
    p, f = _dev(pos), _dev(freq)
    spp.spp_rotary_table(p.data_ptr(), T + 3, axes, axis_of, f.data_ptr(), T, table.data_ptr(), _stream())
    torch.cuda.synchronize()
    got = _host(table)
    want = oa.rotary_table(pos[:, :T], axis_of, freq)
    assert np.max(np.abs(got[:T] - want)) <= 4 * U32
    assert np.all(got[T] == 9.0)


# -------------------------------------------------------------------- store, load

def _store(torch, rng, T, H, Hk, d, page, F, dtype, slots, n_pages, values=None, in_place=False, queries=True):
    """Runs the call on rows of one fused product; returns (device cache, oracle cache, q_out, wanted q)."""
    from paper_2607_24787_amd import spp
    desc = spp.make_attn_desc(H, Hk, d, page, n_pages)
    wide = (H + 2 * Hk) * d + (8 if dtype == "bf16" else 4)
    x = rng.normal(size=(T, wide)).astype(np.float32) if values is None else values
    rows = _dev(x, dtype)
    x = _host(rows)
    table = None
    if F:
        table = _host(_dev(oa.rotary_table(rng.integers(0, 5000, size=(1, T)), [0] * F, 1e4 ** (-np.arange(F) / F)).astype(np.float32)))
    raw = rng.integers(0, 256, size=(n_pages, Hk, page * (d + d // 16)), dtype=np.uint8)
    ora = oa.Cache(Hk, d, page, n_pages, raw)
    cache, tab = _dev(raw), _dev(table) if F else None
    size = rows.element_size()
    q_out = rows if in_place else torch.full((T + 1, H * d), 5.0, device="cuda", dtype=rows.dtype)
    q_stride = wide if in_place else H * d
    at = rows.data_ptr()
    s = _dev(np.asarray(slots, dtype=np.int64))
    heads = x[:, :(H + 2 * Hk) * d].reshape(T, -1, d)
    spp.spp_kv4_store(desc, cache.data_ptr(), _code(dtype), at if queries else 0, wide if queries else 0, q_out.data_ptr() if queries else 0, q_stride,
                      at + H * d * size, wide, at + (H + Hk) * d * size, wide, tab.data_ptr() if F else 0, F, s.data_ptr(), T,
                      _stream())
    torch.cuda.synchronize()
    with np.errstate(all="ignore"):
        want_q = oa.store(ora, heads[:, :H], heads[:, H:H + Hk], heads[:, H + Hk:], table, slots)
    want_q = _host(torch.from_numpy(want_q).to(rows.dtype))
    if not in_place and queries:
        assert bool((q_out[T] == 5.0).all())
    got_q = _host(q_out)[:T, :H * d].reshape(T, H, d) if queries else want_q
    return cache, ora, got_q, want_q, rows, x


STORES = [(1, 32, 4, 128, 64, 64, "bf16"), (1, 1, 1, 64, 16, 0, "f32"), (3, 8, 8, 64, 16, 32, "bf16"),
          (37, 5, 1, 128, 32, 16, "f32"), (130, 6, 2, 64, 256, 24, "bf16"), (70, 4, 4, 128, 16, 40, "f32"),
          (5, 40, 8, 128, 128, 0, "bf16")]


@pytest.mark.parametrize("T,H,Hk,d,page,F,dtype", STORES)
@pytest.mark.parametrize("in_place", [False, True])
def test_store_writes_the_plain_forms_bytes(torch, T, H, Hk, d, page, F, dtype, in_place):
    rng = np.random.default_rng(T + d)
    n_pages = -(-T // page) + 2
    slots = rng.permutation(n_pages * page)[:T]
    cache, ora, q, want_q, rows, x = _store(torch, rng, T, H, Hk, d, page, F, dtype, slots, n_pages, in_place=in_place)
    assert np.array_equal(cache.cpu().numpy(), ora.raw)
    assert np.array_equal(q, want_q)
    if in_place:   # the rest of the rows stays
        assert np.array_equal(_host(rows)[:, H * d:], x[:, H * d:])


def test_store_keys_and_values_alone(torch):
    rng = np.random.default_rng(2)
    cache, ora, _, _, _, _ = _store(torch, rng, 9, 4, 2, 64, 16, 32, "bf16", np.arange(9) + 3, 1, queries=False)
    assert np.array_equal(cache.cpu().numpy(), ora.raw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_store_of_every_kind_of_value(torch, dtype):
    """Ties, zeros of both signs, values next to the borders of scales, extremes, infinities and NaN; no rotation, so that
    each value reaches the quantiser as it is."""
    rng = np.random.default_rng(3)
    H, Hk, d, T = 2, 2, 64, 64
    x = rng.normal(size=(T, (H + 2 * Hk) * d + (8 if dtype == "bf16" else 4))).astype(np.float32)
    mags = np.array([0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7], dtype=np.float32)
    for t in range(T):
        pick = mags[rng.integers(0, 16, size=x.shape[1])] * rng.choice([-1, 1], size=x.shape[1])
        if t < 40:
            with np.errstate(all="ignore"):
                x[t] = (pick * np.float32(2.0) ** rng.integers(-130, 126)).astype(np.float32)
        elif t < 44:
            x[t] = 0.0 * pick
        elif t < 48:
            x[t, rng.integers(0, x.shape[1])] = np.inf
        elif t < 52:
            x[t, rng.integers(0, x.shape[1])] = np.nan
        elif t < 56:
            x[t] = rng.choice([3e38, -3.3e38, 1e38], size=x.shape[1])
        elif t < 60:
            x[t] = rng.choice([1e-45, -1e-40, 1e-38, 0], size=x.shape[1])
        else:
            x[t] = np.nextafter(pick, np.float32(9) * np.sign(pick))
    cache, ora, q, want_q, _, _ = _store(torch, rng, T, H, Hk, d, 16, 0, dtype, np.arange(T), 4, values=x)
    assert np.array_equal(cache.cpu().numpy(), ora.raw)
    assert np.array_equal(q, want_q, equal_nan=True)


def test_store_skips_slots_outside_and_repeats_stay_in_their_slot(torch):
    rng = np.random.default_rng(4)
    slots = np.array([-1, 31, 32, 1 << 40, -(1 << 62), 0, (1 << 63) - 1])
    cache, ora, q, want_q, _, _ = _store(torch, rng, 7, 4, 2, 64, 16, 32, "bf16", slots, 2)
    assert np.array_equal(cache.cpu().numpy(), ora.raw)      # the oracle's write() skips them too
    assert np.array_equal(q, want_q)                         # their queries turn all the same
    cache, ora, _, _, _, _ = _store(torch, rng, 6, 4, 2, 64, 16, 0, "bf16", np.array([3, 9, 3, 3, 9, 20]), 2)
    got = oa.Cache(2, 64, 16, 2, cache.cpu().numpy())
    for slot in set(range(32)) - {3, 9}:
        for kv in range(2):
            assert all(np.array_equal(a, b) for a, b in zip(got.codes(kv, slot), ora.codes(kv, slot)))


@pytest.mark.parametrize("T,Hk,d,page,dtype", [(1, 1, 64, 16, "bf16"), (45, 4, 128, 16, "f32"), (300, 3, 64, 64, "f32"),
                                               (77, 8, 128, 256, "bf16")])
@pytest.mark.parametrize("which", ["kv", "k", "v"])
def test_load(torch, T, Hk, d, page, dtype, which):
    from paper_2607_24787_amd import spp
    rng = np.random.default_rng(T)
    n_pages = 3 + T // page
    raw = rng.integers(0, 256, size=(n_pages, Hk, page * (d + d // 16)), dtype=np.uint8)
    raw[:, :, page * d:] = rng.choice([2, 3, 60, 127, 130, 251, 252, 255], size=raw[:, :, page * d:].shape)
    ora = oa.Cache(Hk, d, page, n_pages, raw)
    slots = rng.integers(0, n_pages * page, size=T)
    if T > 1:
        slots[:2] = [-3, n_pages * page]
    cache, s = _dev(raw), _dev(slots.astype(np.int64))
    wide = Hk * d + 8
    outs = [torch.full((T, wide), 3.0, device="cuda", dtype=torch.bfloat16 if dtype == "bf16" else torch.float32) for _ in "kv"]
    desc = spp.make_attn_desc(Hk * 2, Hk, d, page, n_pages)
    spp.spp_kv4_load(desc, cache.data_ptr(), _code(dtype), s.data_ptr(), T, outs[0].data_ptr() if "k" in which else 0, wide,
                     outs[1].data_ptr() if "v" in which else 0, wide, _stream())
    torch.cuda.synchronize()
    for kv, out in enumerate(outs):
        want = np.full((T, wide), 3.0)
        if "kv"[kv] in which:
            for t, slot in enumerate(slots):
                if 0 <= slot < n_pages * page:
                    want[t, :Hk * d] = ora.read(kv, slot).reshape(-1)
        assert np.array_equal(_host(out).astype(np.float64), want, equal_nan=True)


# ---------------------------------------------------------------------- attention

LENGTHS = [1, 0, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 129, 257]
SHAPES = [(8, 1, 128, 16, "bf16"), (32, 4, 128, 64, "bf16"), (3, 3, 64, 32, "bf16"), (5, 1, 64, 16, "f32"),
          (8, 2, 128, 128, "f32"), (16, 1, 64, 256, "bf16"), (24, 1, 128, 32, "f32")]


@pytest.mark.parametrize("heads,kv_heads,d,page,dtype", SHAPES)
def test_decode_one_token_each(torch, heads, kv_heads, d, page, dtype):
    s = Setup([1] * len(LENGTHS), LENGTHS, heads, kv_heads, d, page, dtype, extra_rows=0)
    s.check(s.run(null_start=True))
    s.check(s.run(causal=False), causal=False)


@pytest.mark.parametrize("heads,kv_heads,d,page,dtype", SHAPES)
@pytest.mark.parametrize("causal", [True, False])
def test_a_few_tokens_each(torch, heads, kv_heads, d, page, dtype, causal):
    nq = [3, 1, 0, 5, 2, 4, 9, 33, 7]
    kv = [40, 0, 33, 5, 1, 3, 64, 95, 131]     # more queries than tokens: rows that see nothing
    s = Setup(nq, kv, heads, kv_heads, d, page, dtype, seed=1)
    s.check(s.run(causal=causal), causal=causal)


@pytest.mark.parametrize("d,dtype,page", [(128, "bf16", 16), (64, "f32", 64), (128, "f32", 32), (64, "bf16", 256)])
def test_prompts(torch, d, dtype, page):
    s = Setup([190, 130, 1], [190, 333, 50], 4, 2, d, page, dtype, seed=2)
    s.check(s.run())


@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "f32"), (128, "f32"), (64, "bf16")])
@pytest.mark.parametrize("nq,heads,kv_heads,seqs", [(3, 24, 2, 3), (9, 8, 1, 2), (9, 16, 4, 9), (40, 8, 2, 1), (33, 8, 1, 3)])
def test_every_way_of_cutting_the_work(torch, d, dtype, nq, heads, kv_heads, seqs):
    """Row counts on both sides of each rule, over lengths that are cut into parts, with page tables of pages of 16."""
    kv = [700, 333, 290, 512, 64, 31, 1, 600, 0][:seqs]
    s = Setup([nq] * seqs, kv, heads, kv_heads, d, 16, dtype, seed=nq + seqs)
    for causal in (True, False):
        s.check(s.run(causal=causal), causal=causal)


@pytest.mark.parametrize("seqs,kv_heads", [(65, 1), (200, 2), (300, 4), (1100, 4)])
def test_many_sequences(torch, seqs, kv_heads):
    """More sequences than a wave has lanes, most short, a few long; up to where nothing is split."""
    rng = np.random.default_rng(seqs)
    kv = rng.integers(0, 40, size=seqs)
    kv[rng.integers(0, seqs, size=3)] = [900, 400, 700]
    kv[-1] = 333
    s = Setup([1] * seqs, kv.tolist(), kv_heads * 2, kv_heads, 64, 16, "bf16", seed=seqs, extra_rows=0)
    s.check(s.run(null_start=True))
    nq = rng.integers(0, 4, size=seqs)
    if seqs < 1000:
        s = Setup(nq.tolist(), kv.tolist(), kv_heads * 2, kv_heads, 64, 32, "f32", seed=seqs)
        s.check(s.run())


@pytest.mark.parametrize("T,H", [(1100, 128), (16500, 16)])
def test_store_of_many_queries(torch, T, H):
    """Queries of more than 32 MB go past the caches: the plain form's values all the same."""
    rng = np.random.default_rng(T)
    from paper_2607_24787_amd import spp
    d = 128
    rows = torch.randn((T, (H + 2) * d), device="cuda").bfloat16()
    if T * H * d * 2 <= 32 << 20:
        rows = rows.float()
    code = spp.DTYPE_BF16 if rows.dtype == torch.bfloat16 else spp.DTYPE_F32
    assert T * H * d * rows.element_size() > 32 << 20
    desc = spp.make_attn_desc(H, 1, d, 16, -(-T // 16))
    cache = torch.zeros(spp.spp_kv4_cache_bytes(desc), dtype=torch.uint8, device="cuda")
    table = _dev(oa.rotary_table(rng.integers(0, 9000, size=(1, T)), [0] * 64, 1e4 ** (-np.arange(64) / 64)).astype(np.float32))
    out = torch.empty((T, H * d), device="cuda", dtype=rows.dtype)
    slots = torch.arange(T, device="cuda")
    at, size, wide = rows.data_ptr(), rows.element_size(), (H + 2) * d
    spp.spp_kv4_store(desc, cache.data_ptr(), code, at, wide, out.data_ptr(), H * d, at + H * d * size, wide,
                      at + (H + 1) * d * size, wide, table.data_ptr(), 64, slots.data_ptr(), T, _stream())
    torch.cuda.synchronize()
    want = torch.from_numpy(oa.rotate(_host(rows)[:, :H * d].reshape(T, H, d), _host(table))).to(rows.dtype)
    assert torch.equal(out.cpu().reshape(T, H, d), want)


@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "f32")])
@pytest.mark.parametrize("nq", [1, 3])
def test_long_sequences(torch, d, dtype, nq):
    s = Setup([nq, nq, nq], [5000, 2000, 70], 4, 1, d, 64, dtype, seed=3)
    s.check(s.run())


def test_hints_do_not_change_what_is_right(torch):
    s = Setup([1, 2, 1], [900, 40, 300], 8, 2, 128, 16, "bf16", seed=4)
    for max_kv in (0, 1, 64, 900, 100000):
        s.check(s.run(max_kv=max_kv))
    for max_q in (2, 3, 50):
        s.check(s.run(max_q=max_q))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq", [40, 15, 4])
def test_what_is_not_finite_reaches_only_rows_that_see_it(torch, dtype, d, nq):
    """Key and value blocks of NaN and of scales beyond the format's in the middle of a causal chunk: rows before are
    as without it, rows from there on are NaN (a value block: its elements)."""
    s = Setup([nq, 6, 1], [90, 6, 70], 4, 2, d, 16, dtype, seed=5)    # many rows, 30 of them, a few
    where = [(0, 88, 1, 1, 255), (0, 87, 0, 0, 255), (1, 3, 1, 0, 255), (2, 69, 1, 1, 255)]
    if nq > 20:
        where += [(0, 77, 1, 1, 255), (0, 60, 0, 0, 255)]
    for b, t, head, kv, byte in where:
        slot = int(s.pages[b, t // 16]) * 16 + t % 16
        p, _, places = s.cache._places(kv, slot)
        s.cache.raw[p, head, places[0]] = byte
    want = s.check(s.run())
    first = nq - (90 - min(t for b, t, *_ in where if b == 0))     # the first query that sees one
    assert np.isnan(want[first:nq]).any() and not np.isnan(want[:first]).any()


def test_queries_that_are_not_finite(torch):
    for dtype in ("bf16", "f32"):
        s = Setup([4, 1], [50, 9], 4, 2, 64, 16, dtype, seed=6)
        clean = _host(s.run())
        s.q[1, 2, 5] = float("inf")
        s.q[3, 0, 0] = float("nan")
        s.q[4, 3, 1] = float("-inf")
        got = _host(s.run())
        hit = np.zeros(got.shape[:2], dtype=bool)
        hit[1, 2] = hit[3, 0] = hit[4, 3] = True
        assert np.isnan(got[hit]).all() and np.array_equal(got[~hit], clean[~hit])


def test_large_scores(torch):
    """Scores from -4000 to 4000: the running maximum moves often, most probabilities are 0."""
    for dtype in ("bf16", "f32"):
        s = Setup([5, 1], [700, 300], 4, 2, 128, 32, dtype, seed=7)
        s.q *= 256.0
        s.check(s.run())


def test_pages_that_are_none(torch):
    s = Setup([3, 2, 1], [60, 60, 60], 4, 2, 128, 16, "bf16", seed=8)
    s.pages[0, 3] = -1                   # tokens 48..59: the last token's row and those before it see them
    s.pages[1, 1] = s.n_pages            # one past the last
    s.pages[2, 0] = np.iinfo(np.int32).min
    want = s.check(s.run())
    assert np.isnan(want[:6]).all()
    s = Setup([20, 1], [40, 17], 4, 2, 64, 16, "f32", seed=9)
    s.pages[0, 2] = np.iinfo(np.int32).max    # tokens 32..39: seen by the last eight queries only
    want = s.check(s.run())
    assert np.isnan(want[12:20]).all() and not np.isnan(want[:12]).any() and not np.isnan(want[20]).any()


def test_lengths_out_of_range(torch):
    s = Setup([2, 1, 1], [30, 20, 10], 4, 2, 64, 16, "bf16", seed=10)
    room = s.wide * 16
    lens = [room + 1, -7, np.iinfo(np.int32).max]
    got = _host(s.run(kv_len=lens))
    assert np.isnan(got[:2]).all() and (got[2] == 0).all() and np.isnan(got[3]).all() and (got[4:] == 7).all()


def test_query_offsets_out_of_range_stay_in_the_rows(torch):
    s = Setup([2, 2], [30, 20], 4, 2, 64, 16, "bf16", seed=11, extra_rows=1)
    s.q_start[:] = [-5, 2, 1 << 30]
    s.nq = [7, 3]
    out = s.run(max_q=8)
    s.q_start[:], s.nq = [0, 2, 5], [2, 3]
    s.check(out)
    s.q_start[:] = [3, 1, 0]              # falling: no queries
    assert (_host(s.run(max_q=8)) == 7).all()


def test_strides_and_in_place(torch):
    for dtype in ("bf16", "f32"):
        s = Setup([3, 4, 1], [50, 20, 600], 6, 2, 64, 16, dtype, seed=12)
        row = s.H * s.d
        wide = torch.full((s.T, row + 24), 7.0, device="cuda", dtype=s.q.dtype)
        wide[:, :row] = s.q.flatten(1)
        out = torch.full((s.T, row + 8), 7.0, device="cuda", dtype=s.q.dtype)
        s.run(q=wide, out=out, q_stride=row + 24, out_stride=row + 8)
        plain = s.run()
        assert torch.equal(out[:, :row].reshape(plain.shape), plain) and bool((out[:, row:] == 7).all())
        s.run(q=wide, out=wide, q_stride=row + 24, out_stride=row + 24)
        assert torch.equal(wide[:8, :row].reshape(8, s.H, s.d), plain[:8])


def test_offsets_beyond_32_bits(torch):
    """A cache of 5 GB whose used pages are its last: the same bits as from a small cache."""
    s = Setup([2, 1], [70, 33], 8, 8, 128, 64, "bf16", seed=13)
    want = s.run()
    big = 5 * 10 ** 9 // (8 * 64 * 136)
    cache = torch.zeros((big, 8, 64 * 136), dtype=torch.uint8, device="cuda")
    cache[-s.n_pages:] = _dev(s.cache.raw)
    from paper_2607_24787_amd import spp
    s.desc = spp.make_attn_desc(8, 8, 128, 64, big)
    s.pages = np.where(s.pages >= 0, s.pages + big - s.n_pages, s.pages)
    assert torch.equal(s.run(cache=cache), want)
    # and a store and a load there
    row = torch.randn((1, 8 * 128), device="cuda").bfloat16()
    slot = torch.tensor([big * 64 - 5], device="cuda")
    back = torch.zeros_like(row)
    spp.spp_kv4_store(s.desc, cache.data_ptr(), 1, 0, 0, 0, 0, row.data_ptr(), 1024, row.data_ptr(), 1024, 0, 0,
                      slot.data_ptr(), 1, _stream())
    spp.spp_kv4_load(s.desc, cache.data_ptr(), 1, slot.data_ptr(), 1, back.data_ptr(), 1024, 0, 0, _stream())
    codes, scales = oa.quantise(_host(row).reshape(8, 128))
    assert np.array_equal(_host(back).reshape(8, 128), oa.values(codes, scales))
    assert int(cache[:big - 1 - s.n_pages].max()) == 0


def test_replays_of_a_graph_with_growing_lengths(torch):
    """Store and attention of a decode step captured once; lengths, slots, tables and rows change between the replays."""
    from paper_2607_24787_amd import spp
    H, Hk, d, page, B, steps = 8, 2, 128, 16, 3, 6
    desc = spp.make_attn_desc(H, Hk, d, page, 3 * 40)
    wide, row = (H + 2 * Hk) * d, H * d
    g = torch.Generator(device="cuda").manual_seed(1)
    pages = torch.randperm(120, device="cuda", generator=g).int().reshape(3, 40).contiguous()
    start = torch.tensor([500, 0, 29], device="cuda")
    caches = [torch.zeros(spp.spp_kv4_cache_bytes(desc), dtype=torch.uint8, device="cuda") for _ in range(2)]
    freq = _dev((1e4 ** (-np.arange(64) / 64)).astype(np.float32))
    size = spp.spp_kv4_attend_workspace(desc, B, 1, 640)
    ws = [torch.zeros(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    pos, slots = torch.zeros((3, B), dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int64, device="cuda")
    kv_len, qkv = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros((B, wide), device="cuda", dtype=torch.bfloat16)
    table = [torch.zeros((B, 2, 64), device="cuda") for _ in range(2)]
    q = [torch.zeros((B, row), device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    out = [torch.zeros((B, row), device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    axes = spp.rotary_axes([24, 20, 20], True)

    def step(i):
        st = _stream()
        spp.spp_rotary_table(pos.data_ptr(), B, 3, axes, freq.data_ptr(), B, table[i].data_ptr(), st)
        spp.spp_kv4_store(desc, caches[i].data_ptr(), 1, qkv.data_ptr(), wide, q[i].data_ptr(), row,
                          qkv.data_ptr() + 2 * row, wide, qkv.data_ptr() + 2 * (row + Hk * d), wide, table[i].data_ptr(), 64,
                          slots.data_ptr(), B, st)
        spp.spp_kv4_attend(desc, caches[i].data_ptr(), 1, q[i].data_ptr(), row, 0, kv_len.data_ptr(), pages.data_ptr(), 40,
                           B, B, 1, 640, True, 0.1, out[i].data_ptr(), row, ws[i].data_ptr(), size, st)

    kv_len.fill_(1)
    slots.copy_(torch.arange(B, device="cuda") * page)
    step(0)
    torch.cuda.synchronize()
    caches[0].zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0)
    for t in range(steps):
        at = start + t
        qkv.normal_(generator=g)
        pos.copy_(torch.stack([at, at + 7, at * 2]))
        slots.copy_(pages.gather(1, (at // page)[:, None])[:, 0].long() * page + at % page)
        kv_len.copy_(at + 1)
        graph.replay()
        torch.cuda.synchronize()
        step(1)
        torch.cuda.synchronize()
        assert torch.equal(caches[0], caches[1]), t
        assert torch.equal(out[0], out[1]), t
        assert bool(torch.isfinite(out[0]).all())


def test_two_calls_at_once_and_another_stream(torch):
    """Calls on two streams, each with its own workspace, give what they give alone."""
    a = Setup([1] * 4, [3000, 1, 900, 64], 8, 2, 128, 16, "bf16", seed=14, extra_rows=0)
    b = Setup([5, 7], [2000, 300], 6, 3, 64, 32, "f32", seed=15)
    alone = [a.run(), b.run()]
    streams = [torch.cuda.Stream() for _ in range(2)]
    caches = [_dev(s.cache.raw) for s in (a, b)]
    torch.cuda.synchronize()
    for _ in range(3):
        outs = []
        for s, st, cache in zip((a, b), streams, caches):
            with torch.cuda.stream(st):
                outs.append(s.run(cache=cache, wait=False))
        torch.cuda.synchronize()
        assert torch.equal(outs[0], alone[0]) and torch.equal(outs[1], alone[1])


def test_results_repeat_bit_for_bit(torch):
    s = Setup([1] * 6, [4000, 33, 900, 64, 1, 2500], 8, 1, 128, 64, "bf16", seed=16, extra_rows=0)
    first = s.run()
    for _ in range(5):
        assert torch.equal(s.run(), first)
