"""GPU tests of the gated delta rule where the time axis is cut into segments that are walked side by side (few heads, long sequences), against the
plain implementation in 64 bits.  Tolerances as in test_gpu_gated_delta.py, whose sums these are: a segment's transition is a product of the same
float32 arithmetic and enters once, so errors stay those of a walk in one piece."""
import numpy as np
import pytest

from test_gpu_gated_delta import BF16, F32, _make, _near, _reference, _state, api  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,Hk,Hv,dk,dv,rate", [
    (1, 1024, 1, 1, 128, 128, 0.02), (1, 1025, 1, 2, 64, 64, 0.02), (2, 1700, 1, 1, 40, 24, 0.02), (1, 2111, 1, 2, 128, 256, 0.3),
    (1, 3200, 1, 1, 96, 32, 2e-3), (3, 1090, 1, 1, 1, 1, 0.02),
])
def test_forward_and_backward(api, io, B, L, Hk, Hv, dk, dv, rate):  # noqa: F811
    t = _make(L, (B, L), Hk, Hv, dk, dv, io, gates="io", rate=rate)
    s0, dl = _state(1, B, Hv, dk, dv), _state(2, B, Hv, dk, dv)
    do = _make(9, (B, L), Hk, Hv, dk, dv, io)["v"]
    o, last, saved = api.lrnnx_gated_delta_fwd(**t, s0=s0, return_last_state=True, return_saved=True)
    r = api.lrnnx_gated_delta_bwd(**t, do=do, saved=saved, s0=s0, ds_last=dl, want_ds0=True)
    fwd, bwd = _reference(t, dk ** -0.5, s0, do, dl)
    tol = F32 if io == "f32" else BF16
    _near(o, np.stack([f[0] for f in fwd]), tol, "o")
    _near(last, np.stack([f[1] for f in fwd]), F32, "last state")
    for n in ("dq", "dk", "dv", "dg", "dbeta"):
        _near(r[n], np.stack([b[n] for b in bwd]), tol, n)
    _near(r["ds0"], np.stack([b["ds0"] for b in bwd]), F32, "ds0")


def test_in_bfloat16_without_states(api):  # noqa: F811
    """The shorter arithmetic of results in bfloat16, in segments."""
    t = _make(3, (1, 2000), 1, 2, 128, 128, "bf16", "io", rate=0.01)
    do = _make(4, (1, 2000), 1, 2, 128, 128, "bf16")["v"]
    o, saved = api.lrnnx_gated_delta_fwd(**t, return_saved=True)
    r = api.lrnnx_gated_delta_bwd(**t, do=do, saved=saved)
    fwd, bwd = _reference(t, 128 ** -0.5, None, do)
    _near(o[0], fwd[0][0], BF16, "o")
    for n in r:
        _near(r[n][0], bwd[0][n], BF16, n)
