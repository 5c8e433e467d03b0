"""A context's attention over decode steps: which calls a step serves, what a refused one leaves behind, and layers whose
sequences are long enough to be cut into parts."""
import numpy as np
import pytest

import oracle as o
from oracle import attention as oa
from test_gpu_attention_layers import CASES, SMALL, U32, stack_of  # noqa: F401 (stack_of: the fixture)

pytestmark = pytest.mark.gpu


def _refused(status, call, *args):
    from paper_2607_24787_amd import spp
    with pytest.raises(spp.SppError) as e:
        call(*args)
    assert e.value.status == status


def _state(st):
    """What a refused call leaves as it is: the clock, the caches, the sequences' lengths."""
    from paper_2607_24787_amd import spp
    import torch
    torch.cuda.synchronize()
    at = st.attention
    return (spp.spp_get_clock(st.ctx), [c.cpu().numpy().tobytes() for c in at.caches], at.kv_len.tolist(), at.length.tolist())


@pytest.mark.parametrize("name", ["bf16_b1", "f32_b3"])
def test_a_step_serves_one_call_of_each_layer(stack_of, name):
    from paper_2607_24787_amd import spp
    from workload import gen
    st = stack_of(CASES[name])
    try:
        h0 = gen.hidden_states(st.cfg, tokens=3)
        for t in range(3):
            st.upload_hidden(h0[t], 0)
            st.attention.next_token(st.cfg.batch)
            st.layer(0, 0, 1, 0)
            before = _state(st)
            _refused(spp.SPP_ESTATE, st.layer, 0, 0, 1, 0)
            _refused(spp.SPP_ESTATE, spp.spp_decode_step, st.ctx, st.cfg.L, st.hbuf[1].data_ptr(), st.hbuf[0].data_ptr(),
                     st.hbuf[1].data_ptr() + 4096, st.cfg.batch, st.cfg.K, 0)
            assert _state(st) == before
            st.layer(1, 1, 0, 0)
            _refused(spp.SPP_ESTATE, st.layer, 1, 0, 1, 0)
        # a step that is refused leaves the one before as it is: served here, not yet below
        args = [st.cfg.batch, st.attention.pos.data_ptr(), st.cfg.batch, st.attention.slots.data_ptr(),
                st.attention.kv_len.data_ptr(), st.attention.pages.data_ptr(), 0]
        _refused(spp.SPP_EINVAL, spp.spp_attention_step, st.ctx, *args)
        _refused(spp.SPP_ESTATE, st.layer, 0, 0, 1, 0)
        st.attention.next_token(st.cfg.batch)
        _refused(spp.SPP_EINVAL, spp.spp_attention_step, st.ctx, *args)
        for l in range(st.cfg.L):
            st.layer(l, l % 2, 1 - l % 2, 0)
    finally:
        st.close()


def test_attention_is_set_before_the_first_layer_call(stack_of):
    from paper_2607_24787_amd import spp
    from workload import gen
    st = stack_of(SMALL.with_(attn_heads=0))
    try:
        desc = spp.make_attn_desc(4, 2, 64, 16, 4)
        h0 = gen.hidden_states(st.cfg, tokens=1)
        _refused(spp.SPP_EINVAL, st.step, h0[0], -2)                 # a refused call is none
        st.step(h0[0], 0)
        out = st.download(st.hbuf[st.last_buf])
        _refused(spp.SPP_ESTATE, spp.spp_set_attention, st.ctx, desc, 1, [], 0, 10)
        st.reset()
        st.step(h0[0], 0)                                            # and the context goes on without
        assert np.array_equal(st.download(st.hbuf[st.last_buf]), out)
    finally:
        st.close()


@pytest.mark.parametrize("how", ["step", "step_from", "decode_step_from"])
def test_a_refused_step_leaves_the_sequences_as_they_were(stack_of, how):
    """A step that a layer refuses, and one that is refused before: the next one writes the places they would have."""
    import torch
    from paper_2607_24787_amd import spp
    from workload import gen
    cfg = CASES["bf16_b1"]
    a, b = stack_of(cfg), stack_of(cfg)
    try:
        h0 = gen.hidden_states(cfg, tokens=18)

        def run(st, t, M_max, B=None):
            src = torch.from_numpy(np.ascontiguousarray(h0[t]).view(np.uint8).reshape(-1).copy()).to(st.device)
            call = getattr(st, how)
            return call(h0[t], M_max, B) if how == "step" else call(src.data_ptr(), M_max, B)

        for t in range(18):
            before = _state(a)
            _refused(spp.SPP_EINVAL, run, a, t, -2)
            assert _state(a) == before
            if t % 5 == 0:
                _refused(spp.SPP_EINVAL, run, a, t, 0, cfg.batch + 1)     # the step itself is refused
                assert _state(a) == before
            run(a, t, 1)
            run(b, t, 1)
            assert np.array_equal(a.download(a.hbuf[a.last_buf]), b.download(b.hbuf[b.last_buf])), t
        assert _state(a) == _state(b)
    finally:
        a.close()
        b.close()


ROWS = SMALL.with_(kv_page=64, kv_tokens=900, attn_heads=32, attn_kv_heads=4, head_dim=128, rotary_sections=(24, 20, 20))
MODEL = ROWS.with_(name="attention_model_shape", D=2048, w_std=0.02, batch=64)
LONG = {
    "bf16_b1": (ROWS, [700]),                                # one sequence in parts
    "bf16_b64": (ROWS.with_(batch=64), None),                # a batch of very different lengths
    "f32_b3": (SMALL.with_(dtype="f32", batch=3, kv_tokens=1300, attn_kv_heads=1), [1200, 3, 650]),
    "bf16_joined_apart": (SMALL.with_(kv_tokens=9000, kv_page=256), [8500]),
    "bf16_b64_model_shape": (MODEL, None),
}


def _grow(st, lens, seed=33):
    """Caches of random codes and ordinary scales, as if the sequences had grown to `lens` tokens (None: ragged)."""
    import torch
    at, cfg, rng = st.attention, st.cfg, np.random.default_rng(seed)
    d, page = cfg.head_dim, cfg.kv_page
    lens = lens or np.exp(rng.uniform(0, np.log(cfg.kv_tokens - 10), size=cfg.batch)).astype(int).tolist()
    for c in at.caches:
        raw = rng.integers(0, 256, size=(at.desc.n_pages, cfg.attn_kv_heads, page * (d + d // 16)), dtype=np.uint8)
        raw[:, :, page * d:] = rng.integers(124, 127, size=raw[:, :, page * d:].shape)
        c.copy_(torch.from_numpy(raw.reshape(-1)))
    at.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
    at.length[:] = lens
    return lens


@pytest.mark.parametrize("name", [n for n in LONG if "model" not in n])
def test_layers_over_long_sequences(stack_of, name):
    """The router's input against 64 bits with the bounds of test_layers_against_64_bits; two steps, so that each layer uses
    the workspace and its counters again.  W_o picks an element of the attention's output for each of u's (over thousands of
    them a sum's bound would say nothing)."""
    import torch
    from paper_2607_24787_amd import spp
    from workload import gen
    cfg, lens = LONG[name]
    u, up = (2.0 ** -8, 2.0 ** -16) if cfg.dtype == "bf16" else (U32, U32)   # a stored value's, a probability's rounding
    st = stack_of(cfg)
    try:
        H, Hk, d, B = cfg.attn_heads, cfg.attn_kv_heads, cfg.head_dim, cfg.batch
        lens = np.asarray(_grow(st, lens))
        h0 = gen.hidden_states(cfg, tokens=2)
        axes = spp.rotary_axes(cfg.rotary_sections, cfg.rotary_interleaved)
        F, pages = axes.size, st.attention.pages.cpu().numpy()
        each = H * d // cfg.D
        pick = np.arange(cfg.D) * each + np.arange(cfg.D) % each
        for _, w_o in st.attention.weights:
            one = torch.zeros((cfg.D, H * d))
            one[np.arange(cfg.D), pick] = 1.0
            w_o.copy_(torch.from_numpy(gen.f32_to_bf16_bits(one.numpy()).view(np.int16)) if cfg.dtype == "bf16" else one)
        for t in range(2):
            st.upload_hidden(h0[t], 0)
            st.attention.next_token(B)
            pos = lens + t
            turn = oa.rotary_table(np.stack([pos] * len(cfg.rotary_sections)), axes, gen.rotary_frequencies(cfg))
            turn = (turn[:, 0] + 1j * turn[:, 1])[:, None]
            for l in range(cfg.L):
                h = o.decode(st.download(st.hbuf[l % 2]), cfg.dtype)
                st.layer(l, l % 2, 1 - l % 2, 0)
                x = spp.spp_get_last_router_input(st.ctx, B, cfg.D).astype(np.float64)
                wqkv = o.decode(gen.attention_weights(cfg, l)[0], cfg.dtype)
                xin = h / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + cfg.rms_eps)

                def stored(y, e):  # the storage type's value of y, and what is open of it where y is known to within e
                    if cfg.dtype == "f32":
                        return y, e + U32 * np.abs(y)
                    lo, mid, hi = (o.decode(gen.f32_to_bf16_bits(np.asarray(z, dtype=np.float32)), "bf16")
                                   for z in (y - e, y, y + e))
                    return mid, np.maximum(hi - mid, mid - lo)

                q, e = stored((xin @ wqkv[:H * d].T).reshape(B, H, d),
                              (np.abs(xin) @ np.abs(wqkv[:H * d]).T).reshape(B, H, d) * (cfg.D + 8) * U32)
                z = (q[..., :F] + 1j * q[..., F:2 * F]) * turn
                both = e[..., :F] + e[..., F:2 * F] + 8 * U32 * (np.abs(q[..., :F]) + np.abs(q[..., F:2 * F]))
                q, e = stored(np.concatenate([z.real, z.imag, q[..., 2 * F:]], axis=-1),
                              np.concatenate([both, both, e[..., 2 * F:]], axis=-1))
                cache = oa.Cache(Hk, d, cfg.kv_page, st.attention.desc.n_pages, st.attention.caches[l].cpu().numpy())
                out, spread, reach = oa.attend(cache, q, list(range(B + 1)), pos + 1, pages, True, d ** -0.5, np.zeros((B, H, d)))
                # the caches' codes reach 6 * 2^-1; the steps' own keys are read
                k_most = max([3.0] + [np.abs(cache.read(0, pages[b, i // cfg.kv_page] * cfg.kv_page + i % cfg.kv_page)).max()
                                      for b in range(B) for i in range(lens[b], pos[b] + 1)])
                ds = reach * 2 * (d + 4) * U32 + d ** -0.5 * k_most * e.sum(-1)
                err = (up + 2 * (ds * np.exp(2 * ds))[..., None] + (max(pos) + 64) * U32) * spread + u * np.abs(out)
                want_u = h + out.reshape(B, -1)[:, pick]
                err_u = err.reshape(B, -1)[:, pick] + 4 * U32 * np.abs(want_u)
                norm = np.sqrt(np.mean(want_u ** 2, axis=1, keepdims=True) + cfg.rms_eps)
                want = want_u / norm
                size = np.sqrt(np.mean(err_u ** 2, axis=1, keepdims=True)) / norm
                bound = 1.1 * (err_u / norm + np.abs(want) * size) + (cfg.D + 8) * U32 * np.abs(want)
                assert np.all(np.abs(x - want) <= bound), (t, l, np.max(np.abs(x - want) / bound))
                absent = h / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + cfg.rms_eps)
                assert np.any(np.abs(x - absent) > bound)
    finally:
        st.close()


@pytest.mark.parametrize("name", list(LONG))
def test_whole_steps_over_long_sequences_give_the_layers_bits(stack_of, name):
    import torch
    from workload import gen
    cfg, lens = LONG[name]
    a, b = stack_of(cfg), stack_of(cfg)
    try:
        _grow(a, lens), _grow(b, lens)
        h0 = gen.hidden_states(cfg, tokens=3)
        for t in range(3):
            a.step(h0[t], 1)
            src = torch.from_numpy(np.ascontiguousarray(h0[t]).view(np.uint8).reshape(-1).copy()).to(b.device)
            b.decode_step_from(src.data_ptr(), 1)
            got = b.download(b.hbuf[b.last_buf])
            assert np.array_equal(a.download(a.hbuf[a.last_buf]), got), t
            assert np.isfinite(o.decode(got, cfg.dtype)).all()
            assert all(torch.equal(x, y) for x, y in zip(a.attention.caches, b.attention.caches)), t
    finally:
        a.close()
        b.close()
