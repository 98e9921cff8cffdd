"""The native half of the binding for the short causal convolution, the loss over a vocabulary and the clipping of gradients: the same results, bit
for bit, as the general path for the usual forms of a call, and nothing taken that the general path refuses or converts; refusals of the general path."""
import pytest

from test_gpu_binding import api  # noqa: F401
from test_gpu_delta_binding import _both
from test_gpu_short_conv import _in, _make as _conv
from test_gpu_vocab_loss import _make as _vocab

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["bld", "bdl"])
def test_conv(api, layout, io):  # noqa: F811
    import torch
    a, dy, dl = _conv(1, layout, 2, 40, 24, 4, io)
    x, dy, w, b, x0, dl = _in(a["x"], layout, False), _in(dy, layout, False), a["weight"].cuda(), a["bias"].cuda(), a["x0"].cuda(), dl.cuda()
    _both(api, api.lrnnx_short_conv_fwd, x, w, layout=layout)
    _both(api, api.lrnnx_short_conv_fwd, x, w, b, "none", x0, layout=layout, return_last_state=True)
    _both(api, api.lrnnx_short_conv_bwd, x, w, dy, layout=layout)
    _both(api, api.lrnnx_short_conv_bwd, x, w, dy, b, x0=x0, dx_last=dl, want_dx0=True, layout=layout)
    cu = torch.tensor([0, 7, 40], dtype=torch.int64, device="cuda")
    _both(api, api.lrnnx_short_conv_fwd, x[0], w, b, x0=x0, cu_seqlens=cu, layout=layout, return_last_state=True)
    _both(api, api.lrnnx_short_conv_bwd, x[0], w, dy[0], b, x0=x0, cu_seqlens=cu, layout=layout)
    wide = torch.cat([x, x], 2 if layout == "bld" else 1)
    _both(api, api.lrnnx_short_conv_fwd, wide[..., 24:] if layout == "bld" else wide[:, 24:], w, b, layout=layout)
    states = [x0.clone() for _ in range(2)]
    one = x[:, 0] if layout == "bld" else x[:, :, 0]
    y = api._native.lrnnx_short_conv_step((one, w, states[0]), dict(bias=b))
    assert y is not None and torch.equal(y, api.lrnnx_short_conv_step.__wrapped__(one, w, states[1], bias=b)) and torch.equal(*states)
    assert api._native.lrnnx_short_conv_fwd((x, w), dict(out=x.clone())) is None
    assert api._native.lrnnx_short_conv_fwd((x, w.double()), {}) is None


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_vocab(api, io):  # noqa: F811
    h, w, target, dloss = (t.cuda() for t in _vocab(1, 24, 300, 64, io))
    _, lse = _both(api, api.lrnnx_vocab_loss_fwd, h, w, target)
    _both(api, api.lrnnx_vocab_loss_fwd, h.view(2, 12, 64), w, target=target.view(2, 12))
    _both(api, api.lrnnx_vocab_loss_bwd, h, w, target, lse, dloss)
    _both(api, api.lrnnx_vocab_loss_bwd, h, w, target, lse, dloss[:1].expand(24), want_dh=False)
    assert api._native.lrnnx_vocab_loss_fwd((h[:, ::2], w[:, ::2], target), {}) is None
    assert api._native.lrnnx_vocab_loss_bwd((h, w, target, lse, dloss.expand(2, 24)[0].repeat_interleave(2)[::2]), {}) is None


def test_clip(api):  # noqa: F811
    import torch
    grads = [torch.randn(n, device="cuda").to(t) for n, t in ((5, torch.float32), (700, torch.bfloat16), (0, torch.float32), (30, torch.float32))]
    norm = _both(api, api.lrnnx_grad_norm, grads)
    assert torch.equal(api._native.lrnnx_grad_norm((tuple(grads),), {}), norm)
    mine, theirs = [t.clone() for t in grads], [t.clone() for t in grads]
    a, b = api._native.lrnnx_grad_clip((mine, norm, 1.0), {}), api.lrnnx_grad_clip.__wrapped__(theirs, norm, 1.0)
    assert type(a) is type(b) is list and all(p is q for p, q in zip(a, mine)) and all(torch.equal(p, q) for p, q in zip(a, b))
    wide = [torch.zeros(t.shape, device="cuda") for t in grads]
    other = [torch.zeros(t.shape, device="cuda") for t in grads]
    a, b = api._native.lrnnx_grad_clip((grads, norm, 1.0), dict(out=wide)), api.lrnnx_grad_clip.__wrapped__(grads, norm, 1.0, out=other)
    assert all(p is q for p, q in zip(a, wide)) and all(torch.equal(p, q) for p, q in zip(a, b))
    assert api._native.lrnnx_grad_clip((grads + grads[:1], norm, 1.0), {}) is None and api._native.lrnnx_grad_norm((iter(grads),), {}) is None
    assert torch.equal(api.lrnnx_grad_norm(iter(grads)), norm)


def test_refusals(api):  # noqa: F811
    import torch
    a, dy, dl = _conv(1, "bld", 2, 9, 8, 4, "bf16")
    x, w, b, x0 = a["x"].cuda(), a["weight"].cuda(), a["bias"].cuda(), a["x0"].cuda()
    for args, kw, error in [
            ((x, w[:, :1].contiguous()), {}, api.LrnnxError), ((x, torch.zeros(8, 5, device="cuda")), {}, api.LrnnxError), ((x, w.bfloat16()), {}, TypeError),
            ((x.half(), w), {}, TypeError), ((x.transpose(1, 2), w), {}, ValueError), ((x, w), dict(layout="bdl"), ValueError), ((x, w), dict(act="relu"), KeyError),
            ((x, w), dict(bias=b[:7]), ValueError), ((x, w), dict(x0=x0.float()), TypeError), ((x, w), dict(x0=x0[:1]), ValueError), ((x[0], w), {}, ValueError),
            ((x.cpu(), w), {}, TypeError), ((x, w), dict(out=torch.zeros(1, 9, 8, dtype=x.dtype, device="cuda").expand(2, 9, 8)), ValueError),
            ((x, w), dict(cu_seqlens=torch.zeros(3, dtype=torch.int64, device="cuda")), ValueError)]:
        with pytest.raises(error):
            api.lrnnx_short_conv_fwd(*args, **kw)
    with pytest.raises(api.LrnnxError) as e:
        api.lrnnx_short_conv_bwd(x, w, dy.cuda(), workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.code == 3
    h, w, target, dloss = (t.cuda() for t in _vocab(1, 24, 300, 64, "bf16"))
    lse = torch.zeros(24, device="cuda")
    for args, error in [((h, w[:, :60], target), ValueError), ((h, w.float(), target), TypeError), ((h, w, target.int()), TypeError), ((h, w, target[:23]), ValueError),
                        ((h.t(), w, target), ValueError), ((h, w, target.cpu()), TypeError)]:
        with pytest.raises(error):
            api.lrnnx_vocab_loss_fwd(*args)
    for kw, error in [(dict(dloss=dloss.double()), TypeError), (dict(dloss=dloss[:5]), ValueError), (dict(lse=lse.double()), TypeError),
                      (dict(want_dh=False, want_dweight=False), ValueError), (dict(dloss=dloss.repeat_interleave(2)[::2]), ValueError)]:
        with pytest.raises(error):
            api.lrnnx_vocab_loss_bwd(**{**dict(h=h, weight=w, target=target, lse=lse, dloss=dloss), **kw})
    with pytest.raises(api.LrnnxError):
        api.lrnnx_vocab_loss_fwd(h[:0], w, target[:0])
    g, norm = [torch.ones(8, device="cuda"), torch.ones(8, device="cuda")], torch.ones((), device="cuda")
    for f, args, kw, error in [
            (api.lrnnx_grad_norm, ([],), {}, ValueError), (api.lrnnx_grad_norm, ([torch.ones(4, 4, device="cuda").t()[1:]],), {}, ValueError),
            (api.lrnnx_grad_norm, ([torch.ones(4)],), {}, TypeError), (api.lrnnx_grad_norm, ([torch.ones(4, device="cuda").half()],), {}, TypeError),
            (api.lrnnx_grad_clip, (g + g[:1], norm, 1.0), {}, ValueError), (api.lrnnx_grad_clip, (g, norm, 1.0), dict(out=g[:1]), ValueError),
            (api.lrnnx_grad_clip, (g, norm, 1.0), dict(out=[g[0], g[0]]), ValueError), (api.lrnnx_grad_clip, (g, norm.double(), 1.0), {}, TypeError),
            (api.lrnnx_grad_clip, (g, norm, -1.0), {}, api.LrnnxError), (api.lrnnx_grad_clip, (g, norm, float("nan")), {}, api.LrnnxError),
            (api.lrnnx_grad_clip, (g, norm, 1.0), dict(out=[t.bfloat16() for t in g]), TypeError)]:
        with pytest.raises(error):
            f(*args, **kw)
    assert all(bool((t == 1).all()) for t in g)
