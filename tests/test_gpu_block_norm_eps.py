"""GPU tests of the norms around a block away from the usual eps, and with weights that are not finite, on rows that do not fill their wavefronts: lanes
without a part of the row must not enter its sums (with eps = 0 their norm is 0 / 0).

Tolerances as derived in test_gpu_block_norm.py: 5e-6 of the 2-norm in float32, 4e-3 in bfloat16; eps enters one addition and changes none of it."""
import numpy as np
import pytest

from _delta_ref import norm_bwd, norm_fwd
from test_gpu_block_norm import _check, _h, _make, _ref_args, api  # noqa: F401

pytestmark = pytest.mark.gpu
SHAPES = [(5, 96, 1), (5, 96, 2), (4, 96, 3), (300, 771, 3), (3, 40, 5), (2, 8190, 3), (700, 1000, 125), (6, 2560, 4), (3, 64, 64)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("eps", [0.0, 1e-2])
@pytest.mark.parametrize("M,D,groups", SHAPES)
def test_eps(api, io, eps, M, D, groups):  # noqa: F811
    a, dh, dy = _make(D + groups, M, D, io, groups=groups, gate="silu")
    h, y = api.lrnnx_block_norm_fwd(**a, eps=eps)
    rh, ry, _ = norm_fwd(_h(a["x"]), **_ref_args(a), eps=eps)
    _check(h, rh, "h")
    _check(y, ry, "y")
    r = api.lrnnx_block_norm_bwd(dh=dh, dy=dy, **a, eps=eps)
    want = norm_bwd(_h(dh), _h(dy), _h(a["x"]), **_ref_args(a), eps=eps)
    for n in want:
        if eps == 0 and D == groups and n == "dx":               # a norm over one element is its sign: nothing to derive
            assert not bool(r[n].any())
        else:
            _check(r[n], want[n], n)


@pytest.mark.parametrize("scale", [1e-18, 1e-20])
def test_tiny_rows_without_eps(api, scale):  # noqa: F811
    """Means of squares of 1e-36, and of 1e-40, which is subnormal (8 bits are left of it: 4e-3 of the norm)."""
    import torch
    x = torch.randn(4, 96, generator=torch.Generator().manual_seed(1)).cuda()
    _, want = api.lrnnx_block_norm_fwd(x, pre_weight=torch.ones(96, device="cuda"), eps=0.0)
    h, y = api.lrnnx_block_norm_fwd(x * scale, pre_weight=torch.ones(96, device="cuda"), eps=0.0)
    assert bool(torch.isfinite(y).all())
    assert np.linalg.norm(_h(y) - _h(want)) <= (5e-6 if scale > 1e-19 else 4e-3) * np.linalg.norm(_h(want))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("M,D,groups", SHAPES)
@pytest.mark.parametrize("which", ["post_weight", "res_scale"])
def test_an_infinite_weight_stays_in_its_column(api, io, M, D, groups, which):  # noqa: F811
    """h is infinite in the first column alone; the second norm of the row is then 0 elsewhere and 0 times infinity there."""
    import torch
    a, _, _ = _make(D, M, D, io, groups=groups)
    a["x"][:, 0] = 1
    a["res_scale"][0] = 0.5
    a[which][0] = float("inf")
    h, y = api.lrnnx_block_norm_fwd(**a)
    assert bool(torch.isinf(h[:, 0]).all()) and bool(torch.isfinite(h[:, 1:]).all())
    assert bool(torch.isnan(y[:, 0]).all()) and not bool(y[:, 1:].any())
