"""CPU checks: the backward call of the gated delta rule takes what the forward call left by its exact size.  Its layout depends on whether a first
state was given, and on lengths and packing: a buffer of another size is one of another call."""
import pytest

from test_delta_cabi import P, SEQ, WORKSPACE, _call, _fill, api  # noqa: F401

BWD = {**{n: P for n in ("dout", "saved", "dq", "dkey", "dval", "dg", "dbeta", "workspace")}, "workspace_bytes": 1 << 40}


def _saved(api, **over):  # noqa: F811
    return _call(api, "lrnnx_gated_delta_saved_bytes", _fill(api.DeltaFwdArgs, **{**SEQ, "o": P, **over}))


def test_other_sizes_are_refused(api):  # noqa: F811
    need = _saved(api)
    for size in (need - 1, need + 1, need + 256, 1 << 40):
        assert _call(api, "lrnnx_gated_delta_bwd", _fill(api.DeltaBwdArgs, **{**SEQ, **BWD, "saved_bytes": size})) == WORKSPACE, size


def test_a_buffer_of_a_call_with_a_first_state_is_refused_without(api):  # noqa: F811
    for over in (dict(gate_dtype=1), dict(gate_dtype=1, dk=128), dict(gate_dtype=1, cu_seqlens=P)):
        with_state = _saved(api, **over, s0=P)
        assert with_state != _saved(api, **over)
        a = _fill(api.DeltaBwdArgs, **{**SEQ, **BWD, **over, "saved_bytes": with_state})
        assert _call(api, "lrnnx_gated_delta_bwd", a) == WORKSPACE, over


@pytest.mark.parametrize("other", [dict(L=164), dict(B=3), dict(Hv=6), dict(dv=128), dict(dk=128)])
def test_a_larger_call_s_buffer_is_refused(api, other):  # noqa: F811
    size = _saved(api, **other)
    assert size > _saved(api)
    assert _call(api, "lrnnx_gated_delta_bwd", _fill(api.DeltaBwdArgs, **{**SEQ, **BWD, "saved_bytes": size})) == WORKSPACE


@pytest.mark.gpu
def test_gradients_without_the_forward_call_s_first_state_are_refused():
    import torch
    from paper_2602_08810_amd import api
    q, k, v = (torch.randn(1, 70, 1, 64, device="cuda").bfloat16() for _ in range(3))
    g, beta = -torch.rand(1, 70, 1, device="cuda").bfloat16(), torch.rand(1, 70, 1, device="cuda").bfloat16()
    s0 = torch.zeros(1, 1, 64, 64, device="cuda")
    _, saved = api.lrnnx_gated_delta_fwd(q, k, v, g, beta, s0=s0, return_saved=True)
    api.lrnnx_gated_delta_bwd(q, k, v, g, beta, v, saved, s0=s0)
    for other in (saved, torch.cat([saved, saved])):
        with pytest.raises(api.LrnnxError) as e:
            api.lrnnx_gated_delta_bwd(q, k, v, g, beta, v, other)
        assert e.value.code == 3
