"""Range of what the gated delta rule keeps for its backward pass in bfloat16 calls: gradients of any scale, rows of different magnitude side by side,
numbers that are not finite in one row or column.

Tolerances.  The gradients are linear in do, and a power of two passes through every product and rounding unchanged as long as nothing is subnormal: equal
bits.  Rows of different magnitude: an element keeps 11 bits down to 2^-29 of its block's largest, so a row 2^-20 of the largest is as accurate as any
other: its own rounding to bfloat16, 2^-9 at most, and half as much again for the states', E's and Z's: 3e-3 each, held to 6e-3 of the row's norm."""
import numpy as np
import pytest

from _delta_ref import delta_bwd

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    import torch
    assert torch.cuda.is_available()
    from paper_2602_08810_amd import api as _api
    _api.lib()
    return _api


def _inputs(seed, B, L, H, dk, dv):
    import torch
    gen = torch.Generator().manual_seed(seed)
    q, k = (torch.nn.functional.normalize(torch.randn(B, L, H, dk, generator=gen), dim=-1).bfloat16().cuda() for _ in range(2))
    v, do = (torch.randn(B, L, H, dv, generator=gen).bfloat16().cuda() for _ in range(2))
    g = (-0.05 * torch.rand(B, L, H, generator=gen)).bfloat16().cuda()
    beta = torch.rand(B, L, H, generator=gen).bfloat16().cuda()
    return q, k, v, g, beta, do


def _grads(api, q, k, v, g, beta, do):
    _, saved = api.lrnnx_gated_delta_fwd(q, k, v, g, beta, return_saved=True)
    return api.lrnnx_gated_delta_bwd(q, k, v, g, beta, do, saved)


@pytest.mark.parametrize("power", [-70, -20, 40])
@pytest.mark.parametrize("dk,dv", [(128, 128), (64, 32), (40, 72)])
def test_scale_of_the_gradient_does_not_matter(api, power, dk, dv):
    import torch
    *inputs, do = _inputs(1, 2, 150, 3, dk, dv)
    a, b = _grads(api, *inputs, do), _grads(api, *inputs, do * 2.0 ** power)
    for n in ("dq", "dk", "dv", "dg", "dbeta"):
        assert torch.equal(a[n] * 2.0 ** power, b[n]), n


def test_scale_of_the_values_does_not_matter(api):
    import torch
    q, k, v, g, beta, do = _inputs(2, 2, 150, 3, 128, 96)
    a, b = _grads(api, q, k, v, g, beta, do), _grads(api, q, k, v * 2.0 ** 50, g, beta, do)
    assert torch.equal(a["dv"], b["dv"])
    for n in ("dq", "dk", "dg", "dbeta"):
        assert torch.equal(a[n] * 2.0 ** 50, b[n]), n


def test_small_rows_beside_large_ones(api):
    import torch
    q, k, v, g, beta, do = _inputs(3, 1, 130, 2, 128, 128)
    do = do * (2.0 ** -(torch.arange(130, device="cuda") % 21)).to(do.dtype)[None, :, None, None]
    r = _grads(api, q, k, v, g, beta, do)
    host = [t[0].double().cpu().numpy() for t in (q, k, v, g, beta)]
    want = delta_bwd(*host, 128 ** -0.5, do[0].double().cpu().numpy())
    got = r["dq"][0].double().cpu().numpy()
    error = np.linalg.norm(got - want["dq"], axis=-1) / np.linalg.norm(want["dq"], axis=-1)
    assert error.max() < 6e-3


@pytest.mark.parametrize("what", [float("inf"), float("nan")])
def test_a_row_that_is_not_finite_leaves_the_others_of_dq(api, what):
    import torch
    *inputs, do = _inputs(4, 1, 128, 2, 64, 64)
    none, bad = do.clone(), do.clone()
    none[0, 40], bad[0, 40] = 0, what
    a, b = _grads(api, *inputs, none), _grads(api, *inputs, bad)
    others = [t for t in range(128) if t != 40]
    assert torch.equal(a["dq"][0, others], b["dq"][0, others])
    assert not torch.isfinite(b["dq"][0, 40]).all()


@pytest.mark.parametrize("what", [float("inf"), float("nan")])
def test_a_column_that_is_not_finite_leaves_the_others_of_dv(api, what):
    import torch
    *inputs, do = _inputs(5, 1, 128, 2, 64, 64)
    none, bad = do.clone(), do.clone()
    none[0, 70, :, 20], bad[0, 70, :, 20] = 0, what
    a, b = _grads(api, *inputs, none), _grads(api, *inputs, bad)
    others = [c for c in range(64) if c != 20]
    assert torch.equal(a["dv"][..., others], b["dv"][..., others])
    assert not torch.isfinite(b["dv"][0, :71, :, 20]).all()
