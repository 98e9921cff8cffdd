"""GPU tests of the clipping's limits, where a quotient of norms is not a number."""
import math

import pytest

from test_gpu_grad_clip import api  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("norm,most,eps,scale", [(0.0, 0.0, 0.0, 1.0), (0.0, 0.0, 1e-6, 0.0), (0.0, 1.0, 0.0, 1.0), (3.0, 0.0, 0.0, 0.0), (math.inf, 2.0, 0.0, 0.0), (math.inf, math.inf, 0.0, 1.0),
                                                 (5.0, math.inf, 0.0, 1.0), (5.0, 5.0, 0.0, 1.0), (8.0, 2.0, 0.0, 0.25), (math.nan, 1.0, 0.0, math.nan)])
def test_scale(api, norm, most, eps, scale, apart):  # noqa: F811
    import torch
    grads = [torch.full((n,), 4.0, device="cuda").to(t) for n, t in ((3, torch.float32), (9000, torch.bfloat16))]
    out = [torch.empty_like(t) for t in grads] if apart else None
    got = api.lrnnx_grad_clip(grads, torch.full((), norm, device="cuda"), most, eps, out=out)
    assert all(torch.equal(t, torch.full_like(t, 4.0 * scale)) if scale == scale else bool(t.isnan().all()) for t in got)


def test_gradients_of_zeros(api):  # noqa: F811
    import torch
    grads = [torch.zeros(700, device="cuda")]
    api.lrnnx_grad_clip(grads, api.lrnnx_grad_norm(grads), 0.0, 0.0)
    assert not bool(grads[0].any())
