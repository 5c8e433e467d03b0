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
                                                      (16, 1, 128, 32, 1), (8, 1, 64, 64, 2)])
@pytest.mark.parametrize("kv", [[90, 33, 2], [2000, 700, 1300]])
def test_few_rows_keep_sixteen_bits_of_a_probability(torch, heads, kv_heads, d, page, nq, kv):
    """Up to 16 rows of a key/value head: a probability is two bf16 terms, off by 2^-8 of what the first leaves of it, so by
    2^-16; the sum it is divided by is fp32's own.  The output's rounding is then all that bf16 costs."""
    s = Setup([nq] * 3, kv, heads, kv_heads, d, page, "bf16", seed=21)
    got = _host(s.run()).astype(np.float64)
    want, spread, reach = oa.attend(s.cache, _host(s.q), s.q_start, s.kv, s.pages, True, s.scale, np.full(got.shape, 7.0))
    n = max(s.kv)
    rel = 2 * (d + 4) * U32 * reach[..., None] + 8 * U32 + 2 * (n / 4 + 32) * U32 + 2.0 ** -16
    bound = rel * spread + U16 * np.abs(want) * (1 + rel) + (6 * n + 1) * 2.0 ** -126
    off = np.abs(got - want)
    assert np.all(off <= bound), np.max(off / bound)


# ----------------------------------------------------------------------- max_q

@pytest.mark.parametrize("max_kv", [0, 700, 100000])    # whole; parts joined by the last workgroup; by a launch
@pytest.mark.parametrize("heads,kv_heads,d,dtype,max_q,nq", [
    (8, 1, 128, "bf16", 1, [3, 1]), (4, 2, 64, "f32", 3, [8, 9]), (24, 1, 128, "bf16", 1, [2, 4]), (6, 1, 64, "f32", 5, [6, 2]),
    (8, 1, 128, "bf16", 5, [9, 41]), (2, 1, 64, "f32", 50, [51, 300]), (8, 8, 128, "f32", 37, [40, 36]), (8, 8, 64, "bf16", 2, [10, 1])])
def test_tokens_past_max_q_stay_as_they_were(torch, heads, kv_heads, d, dtype, max_q, nq, max_kv):
    """Of each sequence the first max_q queries, at the places that all its queries give them."""
    s = Setup(nq, [700, 333], heads, kv_heads, d, 32, dtype, seed=22)
    within = np.concatenate([np.arange(n) < max_q for n in s.nq] + [np.zeros(s.T - sum(s.nq), dtype=bool)])
    beyond = torch.from_numpy(~within).cuda()
    out = s.run(max_q=max_q, max_kv=max_kv)
    assert bool((out[beyond] == 7.0).all())
    whole = s.run()
    out[beyond] = whole[beyond]
    s.check(out)
    both = s.q.clone()                      # in place: those stay queries
    s.run(q=both, out=both, max_q=max_q, max_kv=max_kv)
    assert torch.equal(both[beyond], s.q[beyond])


# ---------------------------------------------- lengths beyond the page table row

@pytest.mark.parametrize("max_kv", [0, 100000])
@pytest.mark.parametrize("nq,room,over,heads,kv_heads,d,dtype", [
    (16, 1, 14, 4, 2, 64, "bf16"), (20, 1, 2, 2, 2, 64, "bf16"), (20, 1, 3, 3, 3, 128, "f32"), (40, 2, 4, 2, 1, 128, "bf16"),
    (50, 2, 700, 3, 1, 64, "f32"), (400, 20, 9, 1, 1, 64, "bf16")])
def test_queries_of_a_sequence_longer_than_its_pages(torch, nq, room, over, heads, kv_heads, d, dtype, max_kv):
    """room pages of 16 tokens, `over` tokens more: queries that see a token give NaN, also those that would see none if the
    sequence ended with its pages; queries before the first token give zeros."""
    s = Setup([nq, 3], [room * 16, 10], heads, kv_heads, d, 16, dtype, seed=23)
    s.wide, s.pages = room, np.ascontiguousarray(s.pages[:, :room])
    n = room * 16 + over
    got = s.run(kv_len=[n, 10], max_kv=max_kv)
    want = s.check(got, kv_len=[n, 10])
    first = max(0, nq - n)
    assert (want[:first] == 0).all() and np.isnan(want[first:nq]).all() and not np.isnan(want[nq:]).any()
    s.check(s.run(kv_len=[n, 10], causal=False, max_kv=max_kv), causal=False, kv_len=[n, 10])


# ------------------------------------------------------------------ far positions

def test_rotary_table_at_the_ends_of_the_positions(torch):
    """The angle's reduction leaves 4 units of 2^-24 (as near positions have) up to the largest position, and for
    frequencies above 1."""
    from paper_2607_24787_amd import spp
    rng = np.random.default_rng(24)
    T, F = 2000, 16
    pos = rng.integers(-(1 << 31), (1 << 31) - 1, size=(2, T)).astype(np.int32)
    pos[:, :2] = [[(1 << 31) - 1, -(1 << 31)]] * 2
    freq = np.concatenate([rng.uniform(0.1, 1, size=F - 4), [1.0, 2.0, 7.3, 50.0]]).astype(np.float32)
    axis_of = np.arange(F) % 2
    table = torch.empty((T, 2, F), device="cuda")
    p, f = _dev(pos), _dev(freq)
    spp.spp_rotary_table(p.data_ptr(), T, 2, axis_of, f.data_ptr(), T, table.data_ptr(), _stream())
    torch.cuda.synchronize()
    assert np.max(np.abs(_host(table) - oa.rotary_table(pos, axis_of, freq))) <= 4 * U32


# ------------------------------------------------- many steps of one workgroup

LONG = [(1, 4, 1, 64, "f32"), (3, 5, 1, 128, "f32"), (2, 8, 1, 128, "bf16"), (5, 3, 1, 64, "bf16"),          # 16 rows
        (3, 8, 1, 128, "bf16"), (3, 8, 1, 64, "f32"), (4, 6, 1, 128, "f32"), (9, 3, 1, 64, "bf16"),          # 32
        (150, 2, 1, 128, "bf16"), (150, 2, 1, 64, "f32"), (70, 2, 1, 128, "f32"), (300, 1, 1, 64, "bf16")]   # shared operands


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("nq,heads,kv_heads,d,dtype", LONG)
def test_long_runs_of_one_workgroup(torch, nq, heads, kv_heads, d, dtype, causal):
    """A hint of no cached tokens leaves every sequence in one part: 22 to 47 tiles of 32 tokens a workgroup, on shuffled
    pages of 16."""
    s = Setup([nq, nq, 2], [1500, 701, 930], heads, kv_heads, d, 16, dtype, seed=25)
    s.check(s.run(causal=causal, max_kv=0), causal=causal)


@pytest.mark.parametrize("max_kv", [0, 1500])
@pytest.mark.parametrize("nq,heads,kv_heads,d,dtype", LONG)
def test_what_is_not_finite_late_in_a_long_run(torch, nq, heads, kv_heads, d, dtype, max_kv):
    """A missing page, a NaN key block and a NaN value block past a workgroup's eighth tile reach the rows that see them, and
    no other."""
    s = Setup([nq, nq, nq], [1500, 701, 930], heads, kv_heads, d, 16, dtype, seed=26)
    s.pages[0, 93] = -1                                                    # tokens 1,488 .. 1,499
    for b, t, kv in ((1, 700 - nq // 2, 0), (2, 929 - nq // 3, 1)):
        slot = int(s.pages[b, t // 16]) * 16 + t % 16
        p, _, places = s.cache._places(kv, slot)
        s.cache.raw[p, 0, places[1 if d == 128 else 0]] = 255
    want = s.check(s.run(max_kv=max_kv))
    assert np.isnan(want[nq - 1]).all() and np.isnan(want[2 * nq - 1]).all() and np.isnan(want[3 * nq - 1]).any()
    assert not np.isnan(want[2 * nq:3 * nq]).all()
    if nq > 12:
        assert not np.isnan(want[0]).any() and not np.isnan(want[nq]).any()


# ------------------------------------------------------------------- one workspace

def test_one_workspace_serves_calls_of_every_shape(torch):
    """Calls of changing head counts, types, lengths and row counts on one workspace, cleared once: the bits of a workspace of
    their own, whatever the calls before have left in it.  Up to 1,024 rows a token."""
    rng = np.random.default_rng(27)
    ws = torch.zeros((1 << 26) + 64, dtype=torch.uint8, device="cuda")
    for heads, kv_heads, d, dtype, seqs, nq in [(8, 1, 128, "bf16", 5, 1), (64, 1, 64, "f32", 3, 1), (32, 4, 128, "bf16", 20, 1),
                                                (6, 3, 64, "bf16", 4, 7), (1024, 1, 64, "bf16", 1, 1), (8, 1, 128, "bf16", 1, 1),
                                                (40, 1, 128, "f32", 2, 2), (4, 2, 64, "f32", 9, 40), (8, 1, 128, "bf16", 5, 1)]:
        kv = [900] + rng.integers(0, 900, size=seqs - 1).tolist()
        s = Setup([nq] * seqs, kv, heads, kv_heads, d, 32, dtype, seed=seqs)
        for max_kv in (900, 100000):
            own = s.run(max_kv=max_kv)
            s.check(own)
            from paper_2607_24787_amd import spp
            size = spp.spp_kv4_attend_workspace(s.desc, seqs, nq, max_kv)
            shared = ws[:size + 64]
            guard = ws[size:size + 64].clone()
            ws[size:size + 64] = 255                 # what run() looks for behind a workspace
            assert torch.equal(s.run(max_kv=max_kv, ws=shared), own)
            ws[size:size + 64] = guard
