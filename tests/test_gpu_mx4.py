"""4-bit matrices on the device against their plain forms (oracle/experts.py).

Bounds.  Stored bytes and loaded values: equal.  Products: the operands are
exact, so an output is off by at most oracle.experts.product's bound (an
addition by at most 2 u32 of the sum of magnitudes, K of them and the joins of
parts), and its rounding (half a step: u16 = 2^-8, u32 = 2^-24 of the value).
"""
import numpy as np
import pytest

from oracle import experts as ox

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def code_of(dtype):
    from paper_2607_24787_amd import spp
    return spp.DTYPE_BF16 if dtype == "bf16" else spp.DTYPE_F32


def stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def host(t):
    import torch
    return t.float().cpu().numpy().astype(np.float64) if t.is_floating_point() else t.cpu().numpy()


def blank(shape, dtype):
    """An output that shows where it was written: NaN, or 0xA5 bytes."""
    import torch
    if dtype == "u8":
        return torch.full(shape, 0xA5, dtype=torch.uint8, device="cuda")
    return torch.full(shape, float("nan"), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")


class Matrix:
    """rows x cols random values in 4 bits: on the device, and as fp64 values."""

    def __init__(self, rng, rows, cols, spread=3, scale=1.0):
        from paper_2607_24787_amd import spp
        x = rng.normal(size=(rows, cols)) * scale * np.exp2(rng.integers(-spread, spread + 1, size=(rows, 1)))
        x = (x.reshape(rows, -1, 32) * np.exp2(rng.integers(-spread, spread + 1, size=(rows, cols // 32, 1)))).reshape(rows, cols)
        self.codes, self.scales = ox.quantise(x.astype(np.float32))
        self.rows, self.cols = rows, cols
        self.upload()

    def upload(self):
        from paper_2607_24787_amd import spp
        self.v = ox.values(self.codes, self.scales)
        self.dev = dev(ox.pack(self.codes)), dev(self.scales)
        self.desc = spp.make_mx4(self.dev[0].data_ptr(), self.dev[1].data_ptr(), self.rows, self.cols)
        return self


# ------------------------------------------------------- quantisation and back

def hard_rows(rows, cols, seed):
    rng = np.random.default_rng(seed)
    x = (rng.normal(size=(rows, cols)) * np.exp(rng.uniform(-30, 30, size=(rows, 1)))).astype(np.float32)
    blocks = x.reshape(-1, 32)
    for i in range(len(blocks)):
        kind = i % 11
        e = 2.0 ** rng.integers(-120, 120)
        if kind == 3:      # ties, borders of scales
            blocks[i, :8] = np.float32(e) * np.array([7.0, -6.0, 5.0, 0.25, 0.75, -1.25, 3.5, 2.5], dtype=np.float32)
            blocks[i, 8:] = 0
        elif kind == 4:
            blocks[i] = 0
            blocks[i, 5] = np.float32(7.0 * e) * np.float32(1 + 2.0 ** -23)
        elif kind == 5:
            blocks[i] = -0.0
        elif kind == 6:
            blocks[i, 31] = [np.inf, -np.inf, np.nan][i % 3]
        elif kind == 7:
            blocks[i] *= np.float32(1e-44) / max(np.abs(blocks[i]).max(), 1e-30)
        elif kind == 8:
            blocks[i] = np.where(rng.random(32) < 0.3, np.finfo(np.float32).max, 1.0)
    return x


@pytest.mark.parametrize("rows,cols,pad", [(1, 32, 0), (1, 2048, 0), (3, 96, 8), (130, 1312, 16), (257, 64, 0), (5, 4096, 24)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantise_and_load(torch, rows, cols, pad, dtype):
    from paper_2607_24787_amd import spp
    x = blank((rows, cols + pad), dtype)
    x[:, :cols] = dev(hard_rows(rows, cols, rows + cols), dtype)
    seen = x[:, :cols].float().cpu().numpy()
    codes, scales = blank((rows * cols // 2 + 64,), "u8"), blank((rows * cols // 32 + 64,), "u8")
    q = spp.make_mx4(codes.data_ptr(), scales.data_ptr(), rows, cols)
    spp.spp_mx4_quantize(code_of(dtype), x.data_ptr(), cols + pad, q, stream())
    want, want_scales = ox.quantise(seen)
    got, got_scales = host(codes), host(scales)
    nan = want_scales == 255
    assert np.array_equal(got_scales[:-64].reshape(rows, -1), want_scales)
    got_codes = ox.unpack(got[:-64].reshape(rows, -1))
    assert np.array_equal(got_codes, want)
    assert (got[-64:] == 0xA5).all() and (got_scales[-64:] == 0xA5).all()
    for to in ("bf16", "f32"):
        out = blank((rows + 1, cols + 8), to)
        spp.spp_mx4_load(q, code_of(to), out.data_ptr(), cols + 8, stream())
        o = host(out)
        assert np.isnan(o[:, cols:]).all() and np.isnan(o[rows]).all()
        v = ox.values(want, want_scales)
        ok = np.repeat(~nan, 32, axis=1)
        assert np.array_equal(o[:rows, :cols][ok], v[ok]) and np.isnan(o[:rows, :cols][~ok]).all()


def test_every_code_and_scale(torch):
    from paper_2607_24787_amd import spp
    codes = np.tile(np.arange(32) % 16, (251, 1)).astype(np.uint8)
    scales = np.arange(2, 253, dtype=np.uint8)[:, None]
    b, s = dev(ox.pack(codes)), dev(scales)
    for dtype in ("bf16", "f32"):
        out = blank((251, 32), dtype)
        spp.spp_mx4_load(spp.make_mx4(b.data_ptr(), s.data_ptr(), 251, 32), code_of(dtype), out.data_ptr(), 32, stream())
        assert np.array_equal(host(out), ox.values(codes, scales))


# -------------------------------------------------------------------- products

def starts(kind, M, G, rng):
    if G == 1:
        return None
    if kind == "even":
        at = np.arange(G + 1) * M // G
    elif kind == "one":      # every row in one group
        at = np.where(np.arange(G + 1) > G // 2, M, 0)
    elif kind == "gaps":     # rows of no group before and after
        cuts = np.sort(rng.integers(1, M - 1, size=G + 1)) if M > 2 else np.full(G + 1, M)
        at = cuts
    else:
        at = np.sort(np.concatenate([[0, M], (M * rng.random(G - 1) ** 2).astype(int)]))
    return at.astype(np.int32)


def check_matmul(rng, M, N, K, G, kind, act, dtype, x_pad=0, out_pad=0, spoil=False):
    from paper_2607_24787_amd import spp
    w = Matrix(rng, G * N, K)
    start = starts(kind, M, G, rng)
    start_dev = None if start is None else dev(start)
    out = blank((M + 1, N + out_pad), dtype)
    args = (G, 0 if start is None else start_dev.data_ptr())
    nan_w = None
    if spoil:   # a NaN block of one weight row of each group
        nan_w = int(rng.integers(0, N))
        w.scales[nan_w::N, int(rng.integers(0, K // 32))] = 255
        w.upload()
    bad_row = int(rng.integers(0, M)) if spoil else None
    if act == "mx4":
        x = Matrix(rng, M, K)
        if spoil:
            x.scales[bad_row, -1] = 255
            x.upload()
        xv = x.v
        spp.spp_mx4_matmul_mx4(w.desc, *args, x.desc, M, code_of(dtype), out.data_ptr(), N + out_pad, stream())
    else:
        x = blank((M, K + x_pad), "bf16")
        x[:, :K] = dev(rng.normal(size=(M, K)) * np.exp(rng.uniform(-3, 3, size=(M, 1))), "bf16")
        if spoil:
            x[bad_row, K - 1] = float("nan")
        xv = host(x[:, :K])
        spp.spp_mx4_matmul(w.desc, *args, x.data_ptr(), K + x_pad, M, code_of(dtype), out.data_ptr(), N + out_pad, stream())
    got = host(out)
    assert np.isnan(got[M]).all() and np.isnan(got[:, N:]).all()
    seen = np.zeros(M, dtype=bool)
    for g, rows in enumerate(ox.groups_of([0, M] if start is None else start, M)):
        seen[rows] = True
        if rows.size == 0:
            continue
        wv = w.v[g * N:(g + 1) * N]
        want, bound = ox.product(xv[rows], wv)
        bound = bound + U[dtype] * (np.abs(want) + bound)
        y = got[rows, :N]
        if spoil:
            nan = np.isnan(want)
            assert nan[:, nan_w].all() and np.array_equal(np.isnan(y), nan)
            y, want, bound = y[~nan], want[~nan], bound[~nan]
        worst = np.max(np.abs(y - want) / bound) if y.size else 0
        assert worst <= 1, (g, worst)
    assert np.isnan(got[:M][~seen]).all()


@pytest.mark.parametrize("act", ["bf16", "mx4"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(1, 1, 32), (1, 16, 64), (1, 5120, 2048), (2, 17, 96), (15, 33, 160), (16, 16, 512), (17, 48, 544),
                                   (33, 100, 1312), (64, 64, 256), (100, 130, 128), (130, 257, 416), (257, 300, 288), (300, 515, 768),
                                   (520, 128, 1024)])
def test_matmul(torch, M, N, K, act, dtype):
    check_matmul(np.random.default_rng(M + N + K), M, N, K, 1, "", act, dtype)


@pytest.mark.parametrize("act", ["bf16", "mx4"])
@pytest.mark.parametrize("M,N,K,G,kind", [
    (1, 20, 64, 3, "one"), (5, 16, 96, 8, "even"), (40, 70, 160, 5, "skewed"), (333, 100, 352, 5, "skewed"), (64, 48, 64, 64, "skewed"),
    (200, 33, 128, 7, "one"), (200, 130, 544, 7, "gaps"), (600, 264, 256, 3, "gaps"), (700, 40, 64, 1024, "skewed"),
    (1100, 140, 320, 4, "skewed")])
def test_matmul_groups(torch, M, N, K, G, kind, act):
    check_matmul(np.random.default_rng(M + N + K + G), M, N, K, G, kind, act, "bf16" if M % 2 else "f32")


@pytest.mark.parametrize("act", ["bf16", "mx4"])
@pytest.mark.parametrize("M,N,K,G,kind", [
    (2500, 3100, 160, 1, ""), (4000, 2100, 2304, 1, ""), (4200, 2050, 1152, 1, ""), (9000, 1030, 64, 1, ""), (5000, 1290, 800, 9, "skewed"),
    (7000, 1000, 1312, 20, "gaps"), (16000, 520, 32, 40, "skewed")])
def test_matmul_of_several_tiles_a_workgroup(torch, M, N, K, G, kind, act):
    check_matmul(np.random.default_rng(M + N + K + G), M, N, K, G, kind, act, "bf16" if N % 4 else "f32")


@pytest.mark.parametrize("act", ["bf16", "mx4"])
@pytest.mark.parametrize("M", [3, 50, 400])
def test_matmul_strides(torch, act, M):
    for x_pad, out_pad, dtype in ((8, 1, "bf16"), (24, 3, "f32"), (0, 2, "bf16"), (64, 8, "bf16"), (8, 4, "f32")):
        check_matmul(np.random.default_rng(M + x_pad), M, 75, 224, 4, "skewed", act, dtype, x_pad, out_pad)


@pytest.mark.parametrize("act", ["bf16", "mx4"])
@pytest.mark.parametrize("M,N,K,G", [(1, 40, 64, 1), (9, 40, 160, 3), (300, 160, 352, 1), (260, 140, 96, 2)])
def test_matmul_what_is_not_finite_stays_in_its_row_and_output(torch, act, M, N, K, G):
    check_matmul(np.random.default_rng(M), M, N, K, G, "even", act, "f32", spoil=True)


def test_matmul_scales_at_both_ends(torch):
    """Scales 2 and 252 against activations whose products stay in range; an infinite activation reaches its row alone."""
    from paper_2607_24787_amd import spp
    for M in (4, 200):
        rng = np.random.default_rng(3)
        for byte, scale in ((2, 2.0 ** 100), (252, 2.0 ** -100)):
            codes = rng.integers(0, 16, size=(64, 128)).astype(np.uint8)
            scales = np.full((64, 4), byte, dtype=np.uint8)
            b, s = dev(ox.pack(codes)), dev(scales)
            x = dev(rng.normal(size=(M, 128)) * scale, "bf16")
            x[2, 7] = float("inf")
            out = blank((M, 64), "f32")
            spp.spp_mx4_matmul(spp.make_mx4(b.data_ptr(), s.data_ptr(), 64, 128), 1, 0, x.data_ptr(), 128, M, spp.DTYPE_F32,
                               out.data_ptr(), 64, stream())
            got, rows = host(out), np.arange(M) != 2
            want, bound = ox.product(host(x)[rows], ox.values(codes, scales))
            assert np.all(np.abs(got[rows] - want) <= bound + U["f32"] * np.abs(want))
            assert not np.isfinite(got[2][(codes[:, 7] & 7) != 0]).any()


def test_matmul_starts_out_of_range_count_as_the_nearest(torch):
    from paper_2607_24787_amd import spp
    rng = np.random.default_rng(4)
    for M in (20, 300):
        w, x = Matrix(rng, 3 * 24, 64), dev(rng.normal(size=(M, 64)), "bf16")
        start = dev(np.array([-7, M // 3, M // 2, M + 1000], dtype=np.int32))
        out = blank((M + 2, 24), "f32")
        spp.spp_mx4_matmul(w.desc, 3, start.data_ptr(), x.data_ptr(), 64, M, spp.DTYPE_F32, out.data_ptr(), 24, stream())
        got = host(out)
        for g, rows in enumerate(ox.groups_of([0, M // 3, M // 2, M], M)):
            want, bound = ox.product(host(x)[rows], w.v[g * 24:g * 24 + 24])
            assert np.all(np.abs(got[rows] - want) <= bound + U["f32"] * np.abs(want))
        assert np.isnan(got[M:]).all()


@pytest.mark.parametrize("act", ["bf16", "mx4"])
def test_matmul_repeats_bit_for_bit_and_in_a_graph(torch, act):
    from paper_2607_24787_amd import spp
    rng = np.random.default_rng(5)
    for M in (7, 330):
        w, start = Matrix(rng, 4 * 40, 352), dev(np.array([0, M // 5, M // 5, M // 2, M], dtype=np.int32))
        x = torch.empty((M, 352), device="cuda", dtype=torch.bfloat16)
        q = torch.zeros((M, 176), device="cuda", dtype=torch.uint8), torch.zeros((M, 11), device="cuda", dtype=torch.uint8)
        m = spp.make_mx4(q[0].data_ptr(), q[1].data_ptr(), M, 352)
        out, eager = blank((M, 40), "f32"), blank((M, 40), "f32")

        def call(to):
            if act == "mx4":
                spp.spp_mx4_quantize(spp.DTYPE_BF16, x.data_ptr(), 352, m, stream())
                spp.spp_mx4_matmul_mx4(w.desc, 4, start.data_ptr(), m, M, spp.DTYPE_F32, to.data_ptr(), 40, stream())
            else:
                spp.spp_mx4_matmul(w.desc, 4, start.data_ptr(), x.data_ptr(), 352, M, spp.DTYPE_F32, to.data_ptr(), 40, stream())

        g = torch.Generator(device="cuda").manual_seed(1)
        x.normal_(generator=g)
        call(eager)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(out)
        for t in range(4):
            x.normal_(generator=g)
            at = np.array([0, t, M // 3, M // 2 + t, M], dtype=np.int32)
            start.copy_(dev(at))
            out.fill_(float("nan"))
            graph.replay()
            call(eager)
            torch.cuda.synchronize()
            # entries that fall back (M = 7, t = 3) name a row twice: it holds no certain result
            times = np.bincount(np.concatenate(ox.groups_of(at, M)), minlength=M)
            assert np.array_equal(host(out)[times == 1], host(eager)[times == 1]) and (times == 1).sum() >= M - 1, t
