"""GPU tests of results in the memory of the convolution's inputs: other channels of the same wider tensor are taken and nothing around them is touched, shifted views are refused."""
import pytest

from test_gpu_short_conv import _in, _make, api  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["bld", "bdl"])
def test_outputs_beside_inputs(api, layout):  # noqa: F811
    import torch
    a, dy, dl = _make(2, layout, 2, 60, 40, 4, "bf16")
    x, dy, w, b, x0, dl = _in(a["x"], layout, False), _in(dy, layout, False), a["weight"].cuda(), a["bias"].cuda(), a["x0"].cuda(), dl.cuda()
    want = api.lrnnx_short_conv_fwd(x, w, b, x0=x0, layout=layout)
    grads = api.lrnnx_short_conv_bwd(x, w, dy, b, x0=x0, dx_last=dl, layout=layout)
    wide = torch.cat([x, dy, torch.zeros_like(x), torch.zeros_like(x)], 2 if layout == "bld" else 1)
    part = lambda i: wide[..., 40 * i:40 * i + 40] if layout == "bld" else wide[:, 40 * i:40 * i + 40]
    api.lrnnx_short_conv_fwd(part(0), w, b, x0=x0, layout=layout, out=part(2))
    r = api.lrnnx_short_conv_bwd(part(0), w, part(1), b, x0=x0, dx_last=dl, layout=layout, out=part(3))
    for i, t in enumerate((x, dy, want, grads["dx"])):
        assert torch.equal(part(i), t), i
    assert torch.equal(r["dweight"], grads["dweight"])


@pytest.mark.parametrize("layout", ["bld", "bdl"])
def test_shifted_views_are_refused(api, layout):  # noqa: F811
    import torch
    room = torch.zeros(2, 61, 49, dtype=torch.bfloat16, device="cuda")
    shape = (2, 60, 40) if layout == "bld" else (2, 40, 48)
    x, w = room[:shape[0], :shape[1], :shape[2]], torch.zeros(40, 4, device="cuda")
    for out in (room[:, 1:1 + shape[1], :shape[2]], room[:, :shape[1], 1:1 + shape[2]], room[:, 1:1 + shape[1], 1:1 + shape[2]]):
        with pytest.raises(api.LrnnxError):
            api.lrnnx_short_conv_fwd(x, w, layout=layout, out=out)
        with pytest.raises(api.LrnnxError):
            api.lrnnx_short_conv_bwd(torch.zeros_like(x), w, x, layout=layout, out=out)
    state = torch.zeros(4, 3, 40, device="cuda")
    with pytest.raises(api.LrnnxError):
        api.lrnnx_short_conv_step(state[:, 0], w, state)
