"""Float32 results of bfloat16 calls of the gated delta rule, against the plain implementation in 64 bits on the same (rounded) inputs.

Tolerance 2e-5 of the 2-norm, as derived for float32 calls: with bfloat16 I/O the inputs are exact factors, and what a float32 result comes from (states,
corrections, decays, sums) is held in 24 bits, whatever the I/O type.  Results rounded to bfloat16: 2^-9 at most, held to 3e-3."""
import numpy as np
import pytest

from test_gpu_gated_delta import F32, _make, _near, _reference, _state, api  # noqa: F401

pytestmark = pytest.mark.gpu
ROUNDED = 3e-3
SHAPES = [  # B, L, Hk, Hv, dk, dv
    (3, 150, 2, 4, 128, 64), (2, 65, 1, 3, 40, 33), (1, 1100, 1, 2, 64, 96), (5, 97, 14, 14, 128, 130), (2, 33, 24, 72, 64, 40), (1, 2100, 1, 1, 128, 128),
    (2, 1, 1, 2, 16, 8), (1, 40, 1, 1, 128, 256),
]


@pytest.mark.parametrize("B,L,Hk,Hv,dk,dv", SHAPES)
@pytest.mark.parametrize("states", [False, True])
def test_gradients_of_float32_gates(api, B, L, Hk, Hv, dk, dv, states):  # noqa: F811
    t = _make(L, (B, L), Hk, Hv, dk, dv, "bf16", rate=0.05)
    do = _make(L + 1, (B, L), Hk, Hv, dk, dv, "bf16")["v"]
    s0, dl = (_state(1, B, Hv, dk, dv), _state(2, B, Hv, dk, dv)) if states else (None, None)
    *_, saved = api.lrnnx_gated_delta_fwd(**t, s0=s0, return_last_state=states, return_saved=True)
    r = api.lrnnx_gated_delta_bwd(**t, do=do, saved=saved, s0=s0, ds_last=dl, want_ds0=states)
    _, bwd = _reference(t, dk ** -0.5, s0, do, dl)
    for n in ("dg", "dbeta") + (("ds0",) if states else ()):
        want = np.stack([b[n] for b in bwd])
        if not want.any():                                       # one step without a state before it: nothing decays
            assert not bool(r[n].any())
            continue
        _near(r[n], want, F32, n)
    for n in ("dq", "dk", "dv"):
        _near(r[n], np.stack([b[n] for b in bwd]), ROUNDED, n)


def test_packed_gradients_of_float32_gates(api):  # noqa: F811
    import torch
    lens, Hk, Hv, dk, dv = [5, 0, 70, 64, 200], 2, 4, 128, 96
    cu = np.concatenate([[0], np.cumsum(lens)])
    t = _make(3, (int(cu[-1]),), Hk, Hv, dk, dv, "bf16", rate=0.05)
    do = _make(4, (int(cu[-1]),), Hk, Hv, dk, dv, "bf16")["v"]
    cut = torch.tensor(cu, dtype=torch.int64, device="cuda")
    _, saved = api.lrnnx_gated_delta_fwd(**t, cu_seqlens=cut, return_saved=True)
    r = api.lrnnx_gated_delta_bwd(**t, do=do, saved=saved, cu_seqlens=cut)
    _, bwd = _reference(t, dk ** -0.5, None, do, None, list(zip(cu[:-1], cu[1:])))
    for n in ("dg", "dbeta"):
        _near(r[n], np.concatenate([b[n] for b in bwd]), F32, n)


@pytest.mark.parametrize("gates", [None, "io"])
@pytest.mark.parametrize("B,L,Hk,Hv,dk,dv", SHAPES)
@pytest.mark.parametrize("last", [False, True])
def test_first_state_s_gradient_without_a_first_state(api, B, L, Hk, Hv, dk, dv, gates, last):  # noqa: F811
    """From a state of zero, with or without a gradient of the last one."""
    t = _make(L + 2, (B, L), Hk, Hv, dk, dv, "bf16", gates, rate=0.05)
    do = _make(L + 3, (B, L), Hk, Hv, dk, dv, "bf16")["v"]
    dl = _state(5, B, Hv, dk, dv) if last else None
    o, s_last, saved = api.lrnnx_gated_delta_fwd(**t, return_last_state=True, return_saved=True)
    r = api.lrnnx_gated_delta_bwd(**t, do=do, saved=saved, ds_last=dl, want_ds0=True)
    fwd, bwd = _reference(t, dk ** -0.5, None, do, dl)
    _near(o, np.stack([f[0] for f in fwd]), ROUNDED, "o")
    _near(s_last, np.stack([f[1] for f in fwd]), F32, "last state")
    _near(r["ds0"], np.stack([b["ds0"] for b in bwd]), F32, "ds0")
    for n in ("dq", "dk", "dv"):
        _near(r[n], np.stack([b[n] for b in bwd]), ROUNDED, n)


@pytest.mark.parametrize("gates", [None, "io"])
def test_last_state_s_gradient_alone(api, gates):  # noqa: F811
    """ds_last without a first state and without its gradient; what was saved without the last state being asked for."""
    B, L, Hk, Hv, dk, dv = 2, 131, 1, 2, 64, 72
    t = _make(7, (B, L), Hk, Hv, dk, dv, "bf16", gates, rate=0.05)
    do, dl = _make(8, (B, L), Hk, Hv, dk, dv, "bf16")["v"], _state(9, B, Hv, dk, dv)
    _, saved = api.lrnnx_gated_delta_fwd(**t, return_saved=True)
    r = api.lrnnx_gated_delta_bwd(**t, do=do, saved=saved, ds_last=dl)
    _, bwd = _reference(t, dk ** -0.5, None, do, dl)
    for n in ("dq", "dk", "dv", "dg", "dbeta"):
        _near(r[n], np.stack([b[n] for b in bwd]), F32 if gates is None and n in ("dg", "dbeta") else ROUNDED, n)
