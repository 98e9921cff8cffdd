"""The native half of the binding for the gated delta rule and the norms around a block: the same results, bit for bit, as the general path for the
usual forms of a call, and nothing taken that the general path refuses or converts."""
import pytest

from test_gpu_binding import api  # noqa: F401
from test_gpu_block_norm import _make as _norm
from test_gpu_gated_delta import _make as _delta, _state

pytestmark = pytest.mark.gpu


def _flat(r):
    return {} if r is None else r if isinstance(r, dict) else dict(enumerate(r if isinstance(r, tuple) else (r,)))


def _both(api, f, *args, **kw):  # noqa: F811
    import torch
    a, b, c = _flat(getattr(api._native, f.__name__)(args, kw)), _flat(f.__wrapped__(*args, **kw)), _flat(f(*args, **kw))
    assert a and list(a) == list(b) == list(c)
    for n in a:
        if a[n] is None:
            assert b[n] is None and c[n] is None
        elif a[n].dtype == torch.uint8:
            assert a[n].shape == b[n].shape
        else:
            assert a[n].dtype == b[n].dtype and a[n].stride() == b[n].stride() and torch.equal(a[n], b[n]) and torch.equal(a[n], c[n]), n
    return f.__wrapped__(*args, **kw)


@pytest.mark.parametrize("io,gates", [("f32", None), ("bf16", None), ("bf16", "io")])
@pytest.mark.parametrize("views", [False, True])
def test_delta(api, io, gates, views):  # noqa: F811
    t = _delta(1, (2, 70), 2, 4, 64, 48, io, gates, views=views)
    s0, dl = _state(2, 2, 4, 64, 48), _state(3, 2, 4, 64, 48)
    do = _delta(4, (2, 70), 2, 4, 64, 48, io)["v"]
    _both(api, api.lrnnx_gated_delta_fwd, **t)
    _both(api, api.lrnnx_gated_delta_fwd, *t.values(), 0.3, s0, return_last_state=True)
    _, saved = _both(api, api.lrnnx_gated_delta_fwd, **t, return_saved=True)
    _both(api, api.lrnnx_gated_delta_bwd, **t, do=do, saved=saved)
    _, _, saved = _both(api, api.lrnnx_gated_delta_fwd, **t, s0=s0, return_last_state=True, return_saved=True)
    _both(api, api.lrnnx_gated_delta_bwd, **t, do=do, saved=saved, s0=s0, ds_last=dl, want_ds0=True)
    one = {n: x[:, 3] for n, x in t.items()}
    states = [s0.clone() for _ in range(2)]
    a = api._native.lrnnx_gated_delta_step((), dict(one, state=states[0]))
    b = api.lrnnx_gated_delta_step.__wrapped__(**one, state=states[1])
    assert a is not None and bool((a == b).all()) and bool((states[0] == states[1]).all())


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("form", [dict(gate="silu"), dict(gate="sigmoid", post="shared", groups=4, residual=None, scale=False, pre=False), dict(residual="io"), dict(post=None)])
def test_norm(api, io, form):  # noqa: F811
    a, dh, dy = _norm(5, 12, 96, io, **form)
    _both(api, api.lrnnx_block_norm_fwd, **a)
    _both(api, api.lrnnx_block_norm_bwd, dh=dh, dy=dy, **a)
    _both(api, api.lrnnx_block_norm_bwd, a.pop("x"), dh, **a)


def test_what_is_left_to_the_general_path(api):  # noqa: F811
    import torch
    t = _delta(6, (8,), 1, 1, 16, 16, "bf16")
    cu = torch.tensor([0, 3, 8], device="cuda")
    n = api._native
    assert n.lrnnx_gated_delta_fwd((), dict(t, cu_seqlens=cu)) is None
    b = {k: x.unsqueeze(0) for k, x in t.items()}
    assert n.lrnnx_gated_delta_fwd((), b) is not None
    for change in (dict(q=b["q"].float()), dict(k=b["k"][:, :5]), dict(g=b["g"].double()), dict(v=b["v"].cpu()), dict(out=torch.empty_like(b["v"])),
                   dict(scale=1), dict(s0=torch.zeros(1, 1, 16, 8, device="cuda")), dict(nonsense=1)):
        assert n.lrnnx_gated_delta_fwd((), {**b, **change}) is None, change
    a, dh, dy = _norm(7, 4, 96, "bf16", gate="silu")
    for change in (dict(groups=5), dict(gate_act=0), dict(eps=1), dict(x=a["x"].t().contiguous().t()), dict(post_weight=a["post_weight"].bfloat16()), dict(out=dh)):
        assert n.lrnnx_block_norm_fwd((), {**a, **change}) is None, change
    assert n.lrnnx_block_norm_bwd((), a) is None
    with pytest.raises(api.LrnnxError):
        api.lrnnx_gated_delta_fwd(*[x[..., :1].expand(1, 8, 1, 200).contiguous() if x.dim() == 4 else x for x in b.values()])
