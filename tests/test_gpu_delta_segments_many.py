"""GPU tests of segments of the time axis with so many heads that a wavefront holds whole columns of a state and the walks that chain segments fill the chip
(the other forms are in test_gpu_delta_segments.py), against the plain implementation in 64 bits.  Tolerances as derived there and for single walks: 2e-5
(float32), 6e-3 (bfloat16) of each tensor's norm."""
import numpy as np
import pytest

from test_gpu_gated_delta import BF16, F32, _make, _near, _reference, _state, api  # noqa: F401

pytestmark = pytest.mark.gpu
SHAPES = [(1, 2570, 24, 24, 16, 64), (1, 2570, 6, 24, 96, 33), (2, 1700, 12, 12, 128, 40)]


def _launches(B, L, Hv, dk, dv):
    """Segments, workgroups of the walks with a wavefront to 16 columns, and of those that find what a segment makes of a state."""
    dvp, dkp, slots = (dv + 31) // 32 * 32, 128 if dk > 64 else 64, (L + 63) // 64
    n = min(256 // (B * Hv * ((dvp + 63) // 64)), slots // 4)
    each = (slots + n - 1) // n
    nseg = (slots + each - 1) // each
    turns = B * Hv * (nseg - 1) * ((dvp + dkp + 63) // 64) / 256
    assert (1 + max(1, turns)) * 2 * each * 1.25 + 2 * nseg + 3 < 2 * slots
    return nseg, B * Hv * nseg * ((dvp + 63) // 64), (B * Hv * (nseg - 1) + 7) // 8 * 8 * (((dvp + dkp) // 16 + 3) // 4)


@pytest.mark.parametrize("io,gates,states", [("f32", None, True), ("f32", None, False), ("bf16", "io", True), ("bf16", "io", False), ("bf16", None, False)])
@pytest.mark.parametrize("B,L,Hk,Hv,dk,dv", SHAPES)
def test_forward_and_backward(api, io, gates, states, B, L, Hk, Hv, dk, dv):  # noqa: F811
    nseg, walks, chains = _launches(B, L, Hv, dk, dv)
    assert nseg >= 3 and walks > 128 and chains > 256
    t = _make(L + dk, (B, L), Hk, Hv, dk, dv, io, gates=gates, rate=0.02)
    s0, dl = (_state(1, B, Hv, dk, dv), _state(2, B, Hv, dk, dv)) if states else (None, None)
    do = _make(9, (B, L), Hk, Hv, dk, dv, io)["v"]
    if states:
        o, last, saved = api.lrnnx_gated_delta_fwd(**t, s0=s0, return_last_state=True, return_saved=True)
    else:
        o, saved = api.lrnnx_gated_delta_fwd(**t, return_saved=True)
    r = api.lrnnx_gated_delta_bwd(**t, do=do, saved=saved, s0=s0, ds_last=dl, want_ds0=states)
    fwd, bwd = _reference(t, dk ** -0.5, s0, do, dl)
    tol = F32 if io == "f32" else BF16
    _near(o, np.stack([f[0] for f in fwd]), tol, "o")
    for n in ("dq", "dk", "dv", "dg", "dbeta"):
        _near(r[n], np.stack([b[n] for b in bwd]), F32 if gates is None and n in ("dg", "dbeta") else tol, n)
    if states:
        _near(last, np.stack([f[1] for f in fwd]), F32, "last state")
        _near(r["ds0"], np.stack([b["ds0"] for b in bwd]), F32, "ds0")
