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
