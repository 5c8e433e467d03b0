"""Attention in front of a context's layers: decode steps of a small stack, layer by layer, against 64 bits.

Per layer call, from the device's own input states and cache bytes: the new
token's cached key and value against the weights' product (no more than one unit
of the block's scale, the half of the format's widest step, and the roundings of
the product away), then the router's input x = rms(u), u = h + W_o o, with o from
the cache as the device holds it.  Bounds per element, u = half a step of the
storage type (2^-8 or 2^-24): a query is rounded twice, its products in fp32 (D
2^-24 relative to sum |W| |x|): rounding is monotone, so a value known to within
s lies between the roundings of its ends, which are mostly one number; with e_q
what is left open of q, a score is off by ds = scale sum e_q |k| + fp32 terms; o
by (u_p + 2 ds + n 2^-24) spread + u |o|, u_p the
rounding of a probability (2^-8 or 2^-24); W_o o by |W_o| times that and K 2^-24
|W_o| |o|; x by the same relative to u's own norm.
"""
import numpy as np
import pytest

import oracle as o
import workload as w
from oracle import attention as oa

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
SMALL = w.MoEConfig(name="attention_small", L=2, D=256, n=16, K=2, I=64, r=8, S=16, windows=(1,), tokens=24, w_std=0.06,
                    attn_heads=4, attn_kv_heads=2, head_dim=64, kv_page=16, kv_tokens=48, rotary_sections=(12, 10, 10), seed=3)
CASES = {
    "f32_b1": SMALL.with_(dtype="f32"),
    "f32_b3": SMALL.with_(dtype="f32", batch=3, attn_heads=3, attn_kv_heads=3),
    "bf16_b1": SMALL,
    "bf16_b4_matrix_cores": SMALL.with_(batch=4, n_shared=1),
    "bf16_b5": SMALL.with_(batch=5, D=272, attn_heads=6, attn_kv_heads=1, rotary_sections=(24,), head_dim=64),
    "bf16_d128_no_rotation": SMALL.with_(head_dim=128, attn_heads=5, attn_kv_heads=5, rotary_sections=(0,)),
}


@pytest.fixture(scope="module")
def stack_of():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_24787_amd.model import OffloadedMoEStack
    return OffloadedMoEStack


@pytest.mark.parametrize("name", list(CASES))
def test_layers_against_64_bits(stack_of, name):
    from paper_2607_24787_amd import spp
    from workload import gen
    cfg = CASES[name]
    u = 2.0 ** -8 if cfg.dtype == "bf16" else U32
    st = stack_of(cfg)
    try:
        H, Hk, d, B = cfg.attn_heads, cfg.attn_kv_heads, cfg.head_dim, cfg.batch
        h0 = gen.hidden_states(cfg, tokens=20)
        axes = spp.rotary_axes(cfg.rotary_sections, cfg.rotary_interleaved)
        freq = gen.rotary_frequencies(cfg)
        rng = np.random.default_rng(1)
        pages = st.attention.pages.cpu().numpy()
        for t in range(20):
            st.upload_hidden(h0[t], 0)
            pos = t + rng.integers(0, 4, size=(len(cfg.rotary_sections), B))
            st.attention.next_token(B, pos)
            table = oa.rotary_table(pos, axes, freq) if axes.size else None
            for l in range(cfg.L):
                src = l % 2
                h = o.decode(st.download(st.hbuf[src]), cfg.dtype)
                st.layer(l, src, 1 - src, 0)
                x = spp.spp_get_last_router_input(st.ctx, B, cfg.D).astype(np.float64)
                wqkv, wo = (o.decode(a, cfg.dtype) for a in gen.attention_weights(cfg, l))
                xin = h / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + cfg.rms_eps)
                qkv = (xin @ wqkv.T).reshape(B, H + 2 * Hk, d)
                slack = (np.abs(xin) @ np.abs(wqkv).T).reshape(B, H + 2 * Hk, d) * (cfg.D + 8) * U32

                def turned(y):
                    if table is None:
                        return y
                    F = axes.size
                    z = (y[..., :F] + 1j * y[..., F:2 * F]) * (table[:, 0] + 1j * table[:, 1])[:, None]
                    return np.concatenate([z.real, z.imag, y[..., 2 * F:]], axis=-1)

                def turned_slack(e, y):  # what an error e of y, and the fp32 products and sums of the turn, may make
                    F = axes.size
                    if table is None:
                        return e
                    both = e[..., :F] + e[..., F:2 * F] + 8 * U32 * (np.abs(y[..., :F]) + np.abs(y[..., F:2 * F]))
                    return np.concatenate([both, both, e[..., 2 * F:]], axis=-1)

                def stored(y, e):  # the storage type's value of y, and what is open of it where y is known to within e
                    if cfg.dtype == "f32":
                        return y, e + U32 * np.abs(y)
                    lo, mid, hi = (o.decode(gen.f32_to_bf16_bits(np.asarray(z, dtype=np.float32)), "bf16")
                                   for z in (y - e, y, y + e))
                    return mid, np.maximum(hi - mid, mid - lo)

                k, v = turned(qkv[:, H:H + Hk]), qkv[:, H + Hk:]
                q, open_q = stored(qkv[:, :H], slack[:, :H])
                q, open_q = stored(turned(q), turned_slack(open_q, q))
                cache = oa.Cache(Hk, d, cfg.kv_page, st.attention.desc.n_pages, st.attention.caches[l].cpu().numpy())
                slots = pages[:, t // cfg.kv_page] * cfg.kv_page + t % cfg.kv_page
                most = np.abs(qkv).max() * 2 + 1
                for b in range(B):
                    for kv, want in ((0, k[b]), (1, v[b])):
                        codes, scales = cache.codes(kv, slots[b])
                        unit = np.repeat(np.ldexp(1.0, scales.astype(int) - 127), 32, axis=-1)
                        off = np.abs(oa.values(codes, scales) - want)
                        assert np.all(off <= unit + 2 * (u * most + slack.max())), (t, l, b, kv)
                out, spread, reach = oa.attend(cache, q, list(range(B + 1)), [t + 1] * B, pages, True, d ** -0.5,
                                               np.zeros((B, H, d)))
                k_most = max(np.abs(cache.read(0, pages[b, i // cfg.kv_page] * cfg.kv_page + i % cfg.kv_page)).max()
                             for b in range(B) for i in range(t + 1))
                ds = reach * 2 * (d + 4) * U32 + d ** -0.5 * k_most * open_q.sum(-1)
                up = 2.0 ** -8 if cfg.dtype == "bf16" else U32
                err = (up + 2 * ds[..., None] + (t + 64) * U32) * spread + u * np.abs(out)
                want_u = h + out.reshape(B, -1) @ wo.T
                err_u = (err.reshape(B, -1) + H * d * U32 * np.abs(out.reshape(B, -1))) @ np.abs(wo).T + 4 * U32 * np.abs(want_u)
                norm = np.sqrt(np.mean(want_u ** 2, axis=1, keepdims=True) + cfg.rms_eps)
                want = want_u / norm
                size = np.sqrt(np.mean(err_u ** 2, axis=1, keepdims=True)) / norm
                bound = 1.1 * (err_u / norm + np.abs(want) * size) + (cfg.D + 8) * U32 * np.abs(want)
                assert np.all(np.abs(x - want) <= bound), (t, l, np.max(np.abs(x - want) / bound))
                # and the bound tells the attention from its absence
                absent = h / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + cfg.rms_eps)
                assert np.any(np.abs(x - absent) > bound)
    finally:
        st.close()


@pytest.mark.parametrize("name", ["f32_b3", "bf16_b1", "bf16_b4_matrix_cores"])
def test_whole_steps_give_the_layers_bits(stack_of, name):
    """spp_decode_step against layer calls one by one, over sequences that grow past a page; a reset starts over."""
    import torch
    from workload import gen
    cfg = CASES[name]
    a, b = stack_of(cfg), stack_of(cfg)
    try:
        h0 = gen.hidden_states(cfg, tokens=20)
        first = None
        for _ in range(2):
            for t in range(20):
                src = torch.from_numpy(np.ascontiguousarray(h0[t]).view(np.uint8).reshape(-1).copy()).to(a.device)
                a.decode_step_from(src.data_ptr(), 1)
                b.step(h0[t], 1)
                got, want = a.download(a.hbuf[a.last_buf]), b.download(b.hbuf[b.last_buf])
                assert np.array_equal(got, want), t
                if t == 19 and first is None:
                    first = got
            assert np.array_equal(got, first)
            a.reset()
            b.reset()
    finally:
        a.close()
        b.close()


def test_refusals_of_the_context_calls(stack_of):
    from paper_2607_24787_amd import spp
    from workload import gen
    st = stack_of(CASES["bf16_b4_matrix_cores"])
    plain = stack_of(SMALL.with_(attn_heads=0))
    proj = stack_of(SMALL.with_(attn_heads=0, has_proj=True))

    def refused(status, call, *args):
        with pytest.raises(spp.SppError) as e:
            call(*args)
        assert e.value.status == status

    try:
        h0 = gen.hidden_states(st.cfg, tokens=1)
        st.upload_hidden(h0[0], 0)
        clock = spp.spp_get_clock(st.ctx)
        refused(spp.SPP_ESTATE, st.layer, 0, 0, 1, 0)            # no step yet
        st.attention.next_token(3)
        refused(spp.SPP_ESTATE, st.layer, 0, 0, 1, 0)            # a step of another batch
        assert spp.spp_get_clock(st.ctx) == clock                # nothing happened
        st.layer(0, 0, 1, 0, B=3)
        desc = st.attention.desc
        refused(spp.SPP_ESTATE, spp.spp_set_attention, st.ctx, desc, 1, [], 0, 10)          # already set
        refused(spp.SPP_EINVAL, spp.spp_set_attention, proj.ctx, desc, 1, [], 0, 10)        # it has the stand-in
        refused(spp.SPP_ESTATE, spp.spp_bind_attention, plain.ctx, 0, 16, 16, 16)
        refused(spp.SPP_ESTATE, spp.spp_attention_step, plain.ctx, 1, 16, 1, 16, 16, 16, 1)
        for change in (dict(axis_of=[0] * 12), dict(axis_of=[1] * 8), dict(n_axes=0), dict(inv_freq_dev=0), dict(max_kv=0),
                       dict(axis_of=[0] * 40), dict(desc=spp.make_attn_desc(64, 64, 128, 16, 4)),
                       dict(desc=spp.make_attn_desc(4, 3, 64, 16, 4))):
            args = dict(desc=desc, n_axes=1, axis_of=[0] * 8, inv_freq_dev=16, max_kv=10)
            refused(spp.SPP_EINVAL, lambda: spp.spp_set_attention(plain.ctx, **{**args, **change}))
        for i in range(3):
            args = [16, 16, 16]
            args[i] = 0
            refused(spp.SPP_EINVAL, spp.spp_bind_attention, st.ctx, 0, *args)
            args[i] = 8
            refused(spp.SPP_EINVAL, spp.spp_bind_attention, st.ctx, 0, *args)
        ok = [3, 16, 4, 16, 16, 16, 1]
        for i, v in ((0, 0), (0, 5), (1, 0), (1, 2), (2, 2), (3, 0), (3, 4), (4, 0), (4, 2), (5, 0), (5, 1), (6, 0), (6, 1 << 40)):
            refused(spp.SPP_EINVAL, spp.spp_attention_step, st.ctx, *[v if k == i else x for k, x in enumerate(ok)])
        for t in range(47):
            st.attention.next_token(3)
        with pytest.raises(ValueError):
            st.attention.next_token(3)                           # the pages are full
    finally:
        for s in (st, plain, proj):
            s.close()
