"""Gradients of the gated delta rule in bfloat16 calls where columns, steps or blocks of steps differ widely in magnitude.

Tolerances.  dv is beta z, element by element, and z keeps 11 bits in a block of 16 columns and at most 32 steps of its own: rounding of both, 2^-9 at most,
held to 6e-3 of each column's (or step's) own norm, like the steps of dq.  Where two halves of a slot do not see each other (a step that forgets everything
between them), each is as accurate as it is alone down to 2^-28 of the other."""
import numpy as np
import pytest

from _delta_ref import delta_bwd
from test_gpu_delta_range import _grads, _inputs, api  # noqa: F401

pytestmark = pytest.mark.gpu


def _want(inputs, do, b=0):
    host = [t[b].double().cpu().numpy() for t in inputs]
    return delta_bwd(*host, inputs[0].shape[-1] ** -0.5, do[b].double().cpu().numpy())


def _errors(got, want, axis):
    got = got.double().cpu().numpy()
    return np.linalg.norm(got - want, axis=axis) / np.linalg.norm(want, axis=axis)


@pytest.mark.parametrize("power", [-25, -45, -80])
@pytest.mark.parametrize("H,dk,dv", [(2, 128, 128), (2, 64, 32), (130, 64, 64)])
def test_small_columns_beside_large_ones(api, power, H, dk, dv):  # noqa: F811
    *inputs, do = _inputs(1, 1, 130, H, dk, dv)
    do[..., 16:32] *= 2.0 ** power
    r, want = _grads(api, *inputs, do), _want(inputs, do)
    assert _errors(r["dv"][0], want["dv"], 0).max() < 6e-3


@pytest.mark.parametrize("power", [-25, -28])
@pytest.mark.parametrize("H,dk,dv", [(2, 128, 128), (2, 64, 32), (130, 64, 64)])
@pytest.mark.parametrize("first", [True, False])
def test_small_steps_beside_large_ones(api, power, H, dk, dv, first):  # noqa: F811
    """One half of a slot of 64 steps is small, and neither half sees the other."""
    *inputs, do = _inputs(2, 1, 128, H, dk, dv)
    inputs[3][:, 32::32] = float("-inf")
    small = slice(0, 32) if first else slice(32, 64)
    do[:, small] *= 2.0 ** power
    r, want = _grads(api, *inputs, do), _want(inputs, do)
    for n in ("dq", "dk", "dv"):
        for part in (slice(0, 32), slice(32, 64), slice(64, 128)):
            got = r[n][0, part].double().cpu().numpy()
            assert np.linalg.norm(got - want[n][part]) < 6e-3 * np.linalg.norm(want[n][part]), (n, part)
    got = r["dbeta"][0, small].double().cpu().numpy()
    assert np.linalg.norm(got - want["dbeta"][small]) < 6e-3 * np.linalg.norm(want["dbeta"][small])
