"""Tokens to their experts and back, and the experts' FFN in 4 bits, on the device against their plain forms.

Bounds.  Sorted pairs and copied rows: equal.  Sums of K rows: each of K + 1
additions and products off by u32 = 2^-24 of the sum of magnitudes, then the
output's rounding (half a step: 2^-8 bf16, 2^-24 fp32).  d_weights: D products
and additions, in parts: (D + 8) u32 of the sum of magnitudes.  The FFN:
oracle.experts.experts, which carries each product's bound through the next
step, and the output's rounding.
"""
import numpy as np
import pytest

from oracle import experts as ox
from tests.test_gpu_mx4 import U, Matrix, blank, code_of, dev, host, stream, torch  # noqa: F401

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24


# ------------------------------------------------------------------------ sort

class Sorted:
    def __init__(self, topk, n, extra=0):
        import torch
        from paper_2607_24787_amd import spp
        T, K = topk.shape
        P = T * K
        self.topk, self.n = dev(topk.astype(np.int32)), n
        self.start = torch.full((n + 2,), -9, dtype=torch.int32, device="cuda")
        self.pair, self.place = (torch.full((P + 1,), -9, dtype=torch.int32, device="cuda") for _ in range(2))
        size = spp.spp_expert_sort_workspace(T, K, n)
        self.space = torch.full((size,), 0x77, dtype=torch.uint8, device="cuda")
        self.call = lambda: spp.spp_expert_sort(self.topk.data_ptr(), T, K, n, self.start.data_ptr(), self.pair.data_ptr(),
                                                self.place.data_ptr(), self.space.data_ptr(), size, stream())
        self.call()


def ids(rng, T, K, n, kind):
    if kind == "distinct":
        logits = rng.normal(size=(T, n)) * 1.5 + rng.normal(size=n)
        return np.argsort(-logits, axis=1)[:, :K]
    if kind == "same":
        return np.full((T, K), n - 1)
    if kind == "bad":
        return rng.integers(-3, n + 3, size=(T, K)) * np.where(rng.random((T, K)) < 0.02, 1 << 20, 1)
    if kind == "none":
        return np.where(rng.random((T, K)) < 0.5, -1, n)
    return rng.integers(0, n, size=(T, K))


@pytest.mark.parametrize("T,K,n,kind", [
    (0, 8, 16, "any"), (1, 1, 1, "any"), (1, 8, 128, "distinct"), (3, 5, 2, "bad"), (64, 8, 128, "distinct"), (63, 1, 64, "any"),
    (65, 1, 65, "same"), (1024, 1, 1024, "any"), (1237, 6, 64, "distinct"), (700, 6, 1000, "bad"), (512, 8, 40, "none"),
    (2000, 8, 128, "bad"), (8192, 8, 128, "distinct"), (5000, 3, 1024, "any"), (9000, 8, 3, "same"), (40000, 8, 96, "bad")])
def test_sort(torch, T, K, n, kind):  # noqa: F811
    topk = ids(np.random.default_rng(T + n), T, K, n, kind)
    s = Sorted(topk, n)
    start, pair, place = ox.sort(topk, n)
    for _ in range(2):
        assert np.array_equal(host(s.start)[:-1], start) and host(s.start)[-1] == -9
        assert np.array_equal(host(s.pair)[:-1], pair) and host(s.pair)[-1] == -9
        assert np.array_equal(host(s.place)[:-1], place) and host(s.place)[-1] == -9
        s.call()


# ------------------------------------------------- rows there, back, gradients

class Routed:
    """Tokens, weights and rows of a sorted routing, with strides of their own."""

    def __init__(self, T, K, n, D, dtype, kind="distinct", pad=8, seed=0):
        rng = np.random.default_rng(seed)
        self.T, self.K, self.D, self.P, self.dtype, self.pad = T, K, D, T * K, dtype, pad
        self.topk = ids(rng, T, K, n, kind)
        self.sorted = Sorted(self.topk, n)
        self.place = ox.sort(self.topk, n)[2].reshape(T, K)
        self.rng = rng
        self.w = dev(rng.normal(size=(T, K)).astype(np.float32))
        self.x, self.y, self.res, self.d_out = (self.rows(r) for r in (T, T * K, T, T))

    def rows(self, r):
        t = blank((r, self.D + self.pad), self.dtype)
        t[:, :self.D] = dev(self.rng.normal(size=(r, self.D)), self.dtype)
        return t

    def of(self, t):
        return host(t[:, :self.D])

    def sum(self, y, w):
        """(sum_k w rows[place], sum of magnitudes), fp64."""
        out, reach = np.zeros((self.T, self.D)), np.zeros((self.T, self.D))
        for k in range(self.K):
            ok = self.place[:, k] >= 0
            term = w[ok, k, None] * y[self.place[ok, k]]
            out[ok] += term
            reach[ok] += np.abs(term)
        return out, reach


SHAPES = [(1, 1, 1, 8, "distinct"), (1, 8, 128, 2048, "distinct"), (5, 3, 7, 24, "bad"), (64, 8, 128, 256, "distinct"),
          (33, 2, 4, 1000, "any"), (257, 6, 64, 1280, "distinct"), (50, 12, 9, 40, "same"), (20, 4, 8, 64, "none"),
          (7, 64, 5, 16, "any"), (3, 2, 5, 4104, "any")]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,K,n,D,kind", SHAPES)
def test_gather_and_combine(torch, T, K, n, D, kind, dtype):  # noqa: F811
    from paper_2607_24787_amd import spp
    r = Routed(T, K, n, D, dtype, kind)
    code, W, place = code_of(dtype), D + r.pad, r.sorted.place.data_ptr()
    rows = blank((r.P + 1, W), dtype)
    spp.spp_expert_gather(code, r.x.data_ptr(), W, place, T, K, D, rows.data_ptr(), W, stream())
    got, named = host(rows), np.zeros(r.P + 1, dtype=bool)
    t, k = np.nonzero(r.place >= 0)
    named[r.place[t, k]] = True
    assert np.array_equal(got[r.place[t, k], :D], r.of(r.x)[t])
    assert np.isnan(got[:, D:]).all() and np.isnan(got[~named]).all()

    for weights in (True, False):
        want, reach = r.sum(r.of(r.y), host(r.w) if weights else np.ones((T, K)))
        for res in (None, "apart", "same"):
            out = blank((T + 1, W), dtype)
            where = r.res
            if res == "same":
                out[:T] = r.res
                where = out
            spp.spp_expert_combine(code, r.y.data_ptr(), W, place, r.w.data_ptr() if weights else 0, T, K, D,
                                   where.data_ptr() if res else 0, W if res else 0, out.data_ptr(), W, stream())
            v = want + (r.of(r.res) if res else 0)
            bound = (K + 2) * U32 * (reach + (np.abs(r.of(r.res)) if res else 0))
            bound = bound + U[dtype] * (np.abs(v) + bound)
            o = host(out)
            assert np.all(np.abs(o[:T, :D] - v) <= bound)
            assert np.isnan(o[:, D:]).all() and np.isnan(o[T]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,K,n,D,kind", SHAPES)
def test_combine_grad(torch, T, K, n, D, kind, dtype):  # noqa: F811
    from paper_2607_24787_amd import spp
    r = Routed(T, K, n, D, dtype, kind, seed=1)
    code, W, place = code_of(dtype), D + r.pad, r.sorted.place.data_ptr()
    y, d, w = r.of(r.y), r.of(r.d_out), host(r.w)
    t, k = np.nonzero(r.place >= 0)
    at = r.place[t, k]
    d_w, w_bound = np.zeros((T, K)), np.zeros((T, K))
    d_w[t, k] = (d[t] * y[at]).sum(1)
    w_bound[t, k] = (D + 8) * U32 * np.abs(d[t] * y[at]).sum(1)
    for weights, rows_too, weights_too, in_place in ((True, True, True, False), (True, True, True, True), (False, True, False, False),
                                                     (True, False, True, False), (True, True, False, False)):
        d_rows = r.y.clone() if in_place else blank((r.P, W), dtype)
        from_rows = d_rows if in_place else r.y
        d_weights = blank((T * K + 1,), "f32")
        spp.spp_expert_combine_grad(code, r.d_out.data_ptr(), W, from_rows.data_ptr() if weights_too else 0, W if weights_too else 0,
                                    place, r.w.data_ptr() if weights else 0, T, K, D, d_rows.data_ptr() if rows_too else 0,
                                    W if rows_too else 0, d_weights.data_ptr() if weights_too else 0, stream())
        if rows_too:
            want = (w[t, k] if weights else np.ones(t.size))[:, None] * d[t]
            got = host(d_rows)
            assert np.all(np.abs(got[at, :D] - want) <= (U32 + U[dtype]) * np.abs(want) * (1 + 1e-6))
            rest = np.setdiff1d(np.arange(r.P), at)
            if in_place:
                assert np.array_equal(got[rest, :D], y[rest])
            else:
                assert np.isnan(got[rest]).all() and np.isnan(got[:, D:]).all()
        if weights_too:
            got = host(d_weights)
            assert np.isnan(got[-1]) and np.all(np.abs(got[:-1].reshape(T, K) - d_w) <= w_bound * (1 + 1e-6))


def test_gradients_against_differences(torch):  # noqa: F811
    """<d_out, combine(rows + e) - combine(rows - e)> / 2 against <d_rows, e>, and so for the weights and the tokens."""
    from paper_2607_24787_amd import spp
    T, K, n, D = 9, 3, 5, 64
    r = Routed(T, K, n, D, "f32", "bad", pad=0, seed=2)
    place, P = r.sorted.place.data_ptr(), T * K
    f32 = spp.DTYPE_F32

    def combine(y, w):
        out = blank((T, D), "f32")
        spp.spp_expert_combine(f32, y.data_ptr(), D, place, w.data_ptr(), T, K, D, 0, 0, out.data_ptr(), D, stream())
        return out.double()

    d_rows, d_w, d_x = torch.zeros((P, D), device="cuda"), torch.zeros((T, K), device="cuda"), blank((T, D), "f32")
    spp.spp_expert_combine_grad(f32, r.d_out.data_ptr(), D, r.y.data_ptr(), D, place, r.w.data_ptr(), T, K, D, d_rows.data_ptr(), D,
                                d_w.data_ptr(), stream())
    spp.spp_expert_combine(f32, r.y.data_ptr(), D, place, 0, T, K, D, 0, 0, d_x.data_ptr(), D, stream())
    g = torch.Generator(device="cuda").manual_seed(0)
    for _ in range(3):
        e_y = torch.empty((P, D), device="cuda").normal_(generator=g)
        e_w = torch.empty((T, K), device="cuda").normal_(generator=g)
        e_x = torch.empty((T, D), device="cuda").normal_(generator=g)
        d = r.d_out.double()
        # combine is linear in each: differences are exact but for rounding.  2 T D sums of K + 2 terms, each within
        # (K + 2) u32 of its magnitudes (at most about 40 here), and twice that much from the inputs' sums
        bound = 2 * T * D * (K + 4) * U32 * 40
        by_rows = (d * (combine(r.y + e_y, r.w) - combine(r.y - e_y, r.w))).sum() / 2
        by_w = (d * (combine(r.y, r.w + e_w) - combine(r.y, r.w - e_w))).sum() / 2
        assert abs(by_rows - (d_rows.double() * e_y).sum()) <= bound
        assert abs(by_w - (d_w.double() * e_w).sum()) <= bound
        # the gather's: <rows' gradient, gather(e_x)> = <d_x, e_x>
        rows = torch.zeros((P, D), device="cuda")
        spp.spp_expert_gather(f32, e_x.data_ptr(), D, place, T, K, D, rows.data_ptr(), D, stream())
        assert abs((rows.double() * r.y.double()).sum() - (d_x.double() * e_x).sum()) <= bound


# ----------------------------------------------------------------- the experts

class Experts:
    def __init__(self, T, n, K, D, I, kind="distinct", seed=0, residual=True, pad=8):
        import torch
        from paper_2607_24787_amd import spp
        rng = np.random.default_rng(seed)
        self.T, self.n, self.K, self.D, self.I, self.pad = T, n, K, D, I, pad
        self.gu = Matrix(rng, n * 2 * I, D, spread=1, scale=1 / np.sqrt(D))
        self.dn = Matrix(rng, n * D, I, spread=1, scale=1 / np.sqrt(I))
        self.topk = ids(rng, T, K, n, kind)
        self.topk_dev = dev(self.topk.astype(np.int32))
        self.gates = dev(rng.random((T, K)).astype(np.float32))
        self.x = blank((T, D + pad), "bf16")
        self.x[:, :D] = dev(rng.normal(size=(T, D)) * 2, "bf16")
        self.res = None
        if residual:
            self.res = blank((T, D + pad), "bf16")
            self.res[:, :D] = dev(rng.normal(size=(T, D)), "bf16")
        self.size = spp.spp_mx4_experts_workspace(n, D, I, T, K)
        self.space = torch.full((self.size + 64,), 0xFF, dtype=torch.uint8, device="cuda")

    def run(self, act, out=None, in_place=False, space=None):
        from paper_2607_24787_amd import spp
        W = self.D + self.pad
        if out is None:
            out = blank((self.T + 1, W), "bf16")
        if in_place:
            out[:self.T] = self.res
        res = out if in_place else self.res
        spp.spp_mx4_experts(self.gu.desc, self.dn.desc, self.n, spp.ACT_MX4 if act == "mx4" else spp.ACT_BF16, self.x.data_ptr(),
                            W, self.topk_dev.data_ptr(), self.gates.data_ptr(), self.T, self.K,
                            0 if res is None else res.data_ptr(), 0 if res is None else W, out.data_ptr(), W,
                            (self.space if space is None else space).data_ptr(), self.size, stream())
        return out

    def check(self, act, out):
        want, bound = ox.experts(host(self.x[:, :self.D]), self.gu.v.reshape(self.n, 2 * self.I, self.D),
                                 self.dn.v.reshape(self.n, self.D, self.I), host(self.topk_dev), host(self.gates),
                                 None if self.res is None else host(self.res[:, :self.D]), act == "mx4")
        bound = bound + U["bf16"] * (np.abs(want) + bound)
        got = host(out)
        worst = np.max(np.abs(got[:self.T, :self.D] - want) / np.maximum(bound, 1e-300))
        assert worst <= 1, worst
        rms = np.sqrt(np.mean((got[:self.T, :self.D] - want) ** 2) / max(np.mean(want ** 2), 1e-300))
        assert rms <= 0.02, rms     # the bound adds up what mostly cancels: a block that went astray shows here
        assert np.isnan(got[:, self.D:][:self.T if self.res is None else 0]).all() and np.isnan(got[self.T]).all()
        assert (host(self.space[self.size:]) == 0xFF).all()


@pytest.mark.parametrize("act", ["bf16", "mx4"])
@pytest.mark.parametrize("T,n,K,D,I,kind", [
    (1, 1, 1, 32, 32, "any"), (1, 128, 8, 256, 96, "distinct"), (1, 64, 6, 1280, 896, "distinct"), (2, 40, 8, 512, 768, "distinct"),
    (3, 8, 2, 96, 64, "any"), (5, 3, 4, 160, 160, "same"), (16, 16, 3, 64, 128, "bad"), (40, 24, 5, 288, 224, "distinct"),
    (64, 40, 8, 256, 128, "distinct"), (130, 8, 2, 320, 96, "any"), (200, 4, 3, 128, 64, "same"), (300, 24, 8, 256, 160, "distinct"),
    (700, 8, 4, 192, 288, "bad"), (3000, 4, 2, 64, 32, "any"), (2500, 200, 4, 32, 64, "same"), (1500, 700, 1, 32, 32, "bad"), (1024, 5, 2, 128, 96, "any"), (33, 6, 64, 64, 32, "any"), (4, 1024, 3, 64, 32, "any"),
    (1, 1, 64, 32, 32, "any"), (1, 1, 64, 448, 32, "any"), (3, 2, 64, 96, 64, "any"), (7, 3, 40, 64, 32, "bad")])
def test_experts(torch, T, n, K, D, I, kind, act):  # noqa: F811
    e = Experts(T, n, K, D, I, kind, seed=T + n, residual=T % 2 == 0)
    e.check(act, e.run(act))


@pytest.mark.parametrize("act", ["bf16", "mx4"])
@pytest.mark.parametrize("T", [1, 6, 90, 600])
def test_experts_in_place_of_their_residual(torch, T, act):  # noqa: F811
    e = Experts(T, 8, 3, 128, 96, seed=5)
    e.check(act, e.run(act, in_place=True))


@pytest.mark.parametrize("act", ["bf16", "mx4"])
@pytest.mark.parametrize("T", [1, 9, 120, 900])
def test_experts_of_no_token(torch, T, act):  # noqa: F811
    """No id in range: the residual, or zeros."""
    for residual in (True, False):
        e = Experts(T, 4, 2, 64, 32, "none", residual=residual)
        got = host(e.run(act))[:T, :64]
        assert np.array_equal(got, host(e.res)[:, :64] if residual else np.zeros((T, 64)))


@pytest.mark.parametrize("act", ["bf16", "mx4"])
@pytest.mark.parametrize("T", [1, 4, 70, 500])
def test_experts_whose_blocks_are_nan_reach_their_tokens_alone(torch, T, act):  # noqa: F811
    e = Experts(T, 6, 2, 96, 64, seed=8)
    e.topk_dev.copy_(dev(np.stack([np.arange(T) % 5, (np.arange(T) + 1) % 5], axis=1).astype(np.int32)))
    if T > 2:
        e.topk_dev[2] = 5
    e.gu.scales[5 * 128:] = 255      # expert 5, which token 2 alone goes to
    e.gu.upload()
    if T > 3:
        e.x[3, 1] = float("inf")
    got = host(e.run(act))
    rows = np.arange(T)
    fine = (rows != 2) & (rows != 3)
    assert np.isfinite(got[:T, :96][fine]).all()
    if T > 2:
        assert np.isnan(got[2, :96]).all()
    if T > 3:
        assert np.isnan(got[3, :96]).any() or np.isinf(got[3, :96]).any()


@pytest.mark.parametrize("act", ["bf16", "mx4"])
def test_one_workspace_over_calls_of_every_size(torch, act):  # noqa: F811
    big = Experts(600, 8, 3, 128, 96, seed=5)
    for T in (600, 1, 90, 3, 600, 20):
        e = Experts(T, 8, 3, 128, 96, seed=T)
        out = e.run(act, space=big.space)
        e.check(act, out)
        assert torch.equal(e.run(act, space=big.space)[:T, :128], out[:T, :128])


@pytest.mark.parametrize("act", ["bf16", "mx4"])
@pytest.mark.parametrize("T", [1, 24, 640])
def test_experts_in_graphs_and_on_a_stream(torch, T, act):  # noqa: F811
    """Two captured calls with a workspace each, replayed side by side with new inputs and eager calls between."""
    es = [Experts(T, 8, 2, 160, 96, seed=s) for s in (1, 2)]
    outs = [blank((T + 1, 168), "bf16") for _ in es]
    streams = [torch.cuda.Stream() for _ in es]
    graphs = []
    torch.cuda.synchronize()
    for e, out, s in zip(es, outs, streams):
        with torch.cuda.stream(s):
            e.run(act, out)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                e.run(act, out)
            graphs.append(graph)
    rng = np.random.default_rng(0)
    for t in range(4):
        for e in es:
            e.x[:, :160] = dev(rng.normal(size=(T, 160)), "bf16")
            e.topk_dev.copy_(dev(ids(rng, T, 2, 8, "bad").astype(np.int32)))
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for e, out in zip(es, outs):
            assert torch.equal(e.run(act)[:T, :160], out[:T, :160]), t
            e.check(act, out)


@pytest.mark.parametrize("T,n,K,D,I", [(1, 8, 2, 64, 32), (50, 16, 4, 256, 96), (400, 8, 3, 128, 160)])
def test_the_operators_together(torch, T, n, K, D, I):  # noqa: F811
    """Sort, gather, product, SwiGLU, product, combine by themselves, against spp_mx4_experts and the plain form; captured too."""
    from paper_2607_24787_amd import spp
    e = Experts(T, n, K, D, I, pad=0, seed=3)
    P, bf16 = T * K, spp.DTYPE_BF16
    s = Sorted(e.topk, n)
    rows, gu = blank((P, D), "bf16"), blank((P, 2 * I), "f32")
    y, out = blank((P, D), "bf16"), blank((T + 1, D), "bf16")

    def chain():
        s.call()
        spp.spp_expert_gather(bf16, e.x.data_ptr(), D, s.place.data_ptr(), T, K, D, rows.data_ptr(), D, stream())
        spp.spp_mx4_matmul(e.gu.desc, n, s.start.data_ptr(), rows.data_ptr(), D, P, spp.DTYPE_F32, gu.data_ptr(), 2 * I, stream())
        h = (torch.nn.functional.silu(gu[:, :I]) * gu[:, I:]).to(torch.bfloat16)
        spp.spp_mx4_matmul(e.dn.desc, n, s.start.data_ptr(), h.data_ptr(), I, P, bf16, y.data_ptr(), D, stream())
        spp.spp_expert_combine(bf16, y.data_ptr(), D, s.place.data_ptr(), e.gates.data_ptr(), T, K, D, e.res.data_ptr(), D,
                               out.data_ptr(), D, stream())

    chain()
    e.check("bf16", out)
    e.check("bf16", e.run("bf16"))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    for t in range(3):
        e.x.normal_()
        s.topk.copy_(s.topk.roll(1, 0))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        chain()
        torch.cuda.synchronize()
        assert torch.equal(got[:T], out[:T]), t
