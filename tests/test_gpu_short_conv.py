"""GPU tests of the short causal convolution against a plain implementation in 64 bits on the same (rounded) inputs.

Tolerances, of the 2-norm of each tensor.  An element of y is five sums of products (2^-24 of their sizes each) and an activation (exponential, sum,
reciprocal, product: 2^-24 each): 9 * 6e-8 = 5e-7, twice that where terms cancel: 1e-6; dx has four such; the weights' gradients add up to some
thousand of them like independent errors, in chains of at most 100: 6e-8 * sqrt(100) + 1e-6, held to 2e-6.  Rounded to bfloat16: at most 2^-8 of
each element, 4e-3; the activation's exponential is then the hardware's (1e-6 of it)."""
import pytest

from _train_ref import conv

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    import torch
    assert torch.cuda.is_available()
    from paper_2602_08810_amd import api as _api
    _api.lib()
    return _api


def _rel(got, want):
    got = got.double().cpu()
    assert got.shape == want.shape
    return ((got - want).norm() / want.norm().clamp(min=1e-300)).item()


def _check(got, want, name):
    import torch
    tol = 4e-3 if got.dtype == torch.bfloat16 else 2e-6 if name in ("dweight", "dbias") else 1e-6
    e = _rel(got, want)
    assert e <= tol, f"{name}: relative error {e:.2e}, tolerance {tol:g}"


def _make(seed, layout, B, L, D, W, io, bias=True, state=True, cu=None):
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    rnd = lambda *s: torch.randn(s, generator=g)
    n = B if cu is None else len(cu) - 1
    a = dict(x=rnd(B, L, D).to(dt), weight=rnd(D, W) * 0.5, bias=rnd(D) * 0.5 if bias else None, x0=rnd(n, W - 1, D).to(dt) if state else None)
    return a, rnd(B, L, D).to(dt), rnd(n, W - 1, D).to(dt) if state else None


def _in(t, layout, packed):
    t = t if layout == "bld" else t.transpose(1, 2).contiguous()
    return (t[0] if packed else t).cuda()


def _out(t, layout, packed):
    t = t.unsqueeze(0) if packed else t
    return t if layout == "bld" else t.transpose(1, 2)


def _both(api, seed, layout, B, L, D, W, io, act="silu", bias=True, state=True, cu=None):
    import torch
    a, dy, dl = _make(seed, layout, B, L, D, W, io, bias, state, cu)
    packed = cu is not None
    leaves = {n: t.double().requires_grad_() for n, t in a.items() if t is not None}
    ref, ref_last = conv(leaves["x"], leaves["weight"], leaves.get("bias"), act, leaves.get("x0"), cu)
    inside = ~torch.isnan(ref)
    outs = ([(ref[inside], dy.double()[inside])] if bool(inside.any()) else []) + ([(ref_last, dl.double())] if state else [])
    grads = torch.autograd.grad([o for o, _ in outs], list(leaves.values()), [d for _, d in outs], allow_unused=True)
    grads = {n: torch.zeros_like(t) if d is None else d for (n, t), d in zip(leaves.items(), grads)}
    opts = dict(bias=None if a["bias"] is None else a["bias"].cuda(), act=act, x0=None if a["x0"] is None else a["x0"].cuda(), layout=layout)
    if packed:
        opts["cu_seqlens"] = torch.tensor(cu, dtype=torch.int64, device="cuda")
    x, w = _in(a["x"], layout, packed), a["weight"].cuda()
    kept = torch.full_like(x, 7.0)
    y, last = api.lrnnx_short_conv_fwd(x, w, return_last_state=True, out=kept, **opts)
    y = _out(y, layout, packed).cpu()
    assert bool((y[~inside] == 7.0).all())
    if bool(inside.any()):
        _check(y[inside], ref.detach()[inside], "y")
    assert torch.equal(last.cpu().double(), ref_last.detach())
    r = api.lrnnx_short_conv_bwd(x, w, _in(dy, layout, packed), dx_last=None if dl is None else dl.cuda(), want_dx0=state, **opts)
    assert set(r) == {"dx", "dweight"} | ({"dbias"} if bias else set()) | ({"dx0"} if state else set())
    for n, t in r.items():
        _check(_out(t, layout, packed) if n == "dx" else t, grads[n[1:]], n)


LAYOUTS, TYPES = ["bld", "bdl"], ["f32", "bf16"]


@pytest.mark.parametrize("io", TYPES)
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("L,D", [(1, 1), (2, 7), (3, 8), (5, 3), (7, 130), (9, 20), (33, 65), (70, 9), (130, 4)])
def test_sizes(api, layout, io, W, L, D):
    _both(api, L * D + W, layout, 2, L, D, W, io)


@pytest.mark.parametrize("io", TYPES)
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("act", ["silu", "none"])
@pytest.mark.parametrize("bias,state", [(True, False), (False, True), (False, False)])
def test_forms(api, layout, io, act, bias, state):
    _both(api, 5, layout, 3, 37, 72, 4, io, act, bias, state)


@pytest.mark.parametrize("io", TYPES)
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("L,D", [(600, 520), (1100, 24), (40, 1100)])
def test_several_tiles_and_workgroups(api, layout, io, L, D):
    _both(api, L, layout, 1, L, D, 4, io)


@pytest.mark.parametrize("io", TYPES)
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("W,D,L,cu", [
    (4, 72, 64, [0, 1, 3, 6, 10, 33, 33, 64]),             # shorter than the filter, without steps, longer
    (3, 5, 41, [0, 20, 41]), (2, 9, 30, [0, 0, 29, 30]),
    (4, 33, 50, [4, 9, 31, 44]),                           # steps before the first and after the last
    (4, 16, 20, [-5, 7, 90]),                              # boundaries beyond the axis
    (4, 8, 12, [12, 12, 12]), (3, 130, 1, [0, 1]), (4, 20, 7, [2, 3])])
def test_packed(api, layout, io, W, D, L, cu):
    for state in (True, False):
        if not state and all(b <= a for a, b in zip(cu, cu[1:])):
            continue
        _both(api, L, layout, 1, L, D, W, io, state=state, cu=cu)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_a_packed_batch_of_many_sequences(api, layout):
    import random
    r = random.Random(3)
    cu = [0]
    for _ in range(90):
        cu.append(cu[-1] + r.choice([0, 1, 2, 3, 5, 8, 13, 40]))
    _both(api, 1, layout, 1, cu[-1] + 3, 20, 4, "f32", cu=cu)


@pytest.mark.parametrize("io", TYPES)
@pytest.mark.parametrize("layout", LAYOUTS)
def test_views_and_outputs_in_views(api, layout, io):
    import torch
    a, dy, dl = _make(9, layout, 2, 45, 51, 4, io)
    w, b, x0 = a["weight"].cuda(), a["bias"].cuda(), a["x0"].cuda()
    x, dy = _in(a["x"], layout, False), _in(dy, layout, False)
    want = api.lrnnx_short_conv_fwd(x, w, bias=b, x0=x0, layout=layout)
    grads = api.lrnnx_short_conv_bwd(x, w, dy, bias=b, x0=x0, dx_last=dl.cuda(), layout=layout)
    def view(t):                                           # a part of the channels and steps of a wider tensor
        wide = torch.zeros(t.shape[0], t.shape[1] + 3, t.shape[2] + 5, dtype=t.dtype, device="cuda")
        v = wide[:, 2:2 + t.shape[1], 1:1 + t.shape[2]]
        v.copy_(t)
        return wide, v
    wide, out = view(torch.zeros_like(x))
    got = api.lrnnx_short_conv_fwd(view(x)[1], w, bias=b, x0=x0, layout=layout, out=out)
    assert got.data_ptr() == out.data_ptr() and torch.equal(out, want)
    out.zero_()
    assert not bool(wide.any())                            # nothing around it was written
    wide, out = view(torch.zeros_like(x))
    r = api.lrnnx_short_conv_bwd(view(x)[1], w, view(dy)[1], bias=b, x0=x0, dx_last=dl.cuda(), layout=layout, out=out)
    assert torch.equal(r["dx"], grads["dx"]) and torch.equal(r["dweight"], grads["dweight"]) and torch.equal(r["dbias"], grads["dbias"])
    out.zero_()
    assert not bool(wide.any())


@pytest.mark.parametrize("io", TYPES)
@pytest.mark.parametrize("W,D", [(2, 1), (3, 9), (4, 64), (4, 771)])
def test_steps_are_the_sequence(api, io, W, D):
    import torch
    a, _, _ = _make(W + D, "bld", 3, 9, D, W, io)
    x, w, b, x0 = (a[n].cuda() for n in ("x", "weight", "bias", "x0"))
    y, last = api.lrnnx_short_conv_fwd(x, w, bias=b, x0=x0, return_last_state=True)
    state = x0.clone()
    for t in range(9):
        step = api.lrnnx_short_conv_step(x[:, t], w, state, bias=b)
        assert _rel(step, y[:, t].double().cpu()) <= (4e-3 if io == "bf16" else 1e-6), t
    assert torch.equal(state, last)
    wide = torch.zeros(D, 2, 3, dtype=x.dtype, device="cuda").permute(2, 0, 1)[:, :, 1]        # neither axis contiguous
    wide.copy_(x[:, 0])
    state, again = x0.clone(), x0.clone()
    want = api.lrnnx_short_conv_step(x[:, 0], w, state, bias=b, act="none")
    assert api.lrnnx_short_conv_step(wide, w, again, bias=b, act="none", out=wide).data_ptr() == wide.data_ptr()
    assert torch.equal(wide, want) and torch.equal(state, again)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_numbers_that_are_not_finite_stay_where_they_belong(api, layout):
    import torch
    cu = [0, 13, 29, 60]
    a, dy, _ = _make(4, layout, 1, 64, 24, 4, "f32", state=False, cu=cu)
    w, b, c = a["weight"].cuda(), a["bias"].cuda(), torch.tensor(cu, dtype=torch.int64, device="cuda")
    run = lambda x, d: (api.lrnnx_short_conv_fwd(_in(x, layout, True), w, bias=b, layout=layout, cu_seqlens=c),
                        api.lrnnx_short_conv_bwd(_in(x, layout, True), w, _in(d, layout, True), bias=b, layout=layout, cu_seqlens=c))
    y, r = run(a["x"], dy)
    x2, dy2 = a["x"].clone(), dy.clone()
    x2[0, 60:], dy2[0, 60:] = float("nan"), float("inf")   # outside every sequence
    y2, r2 = run(x2, dy2)
    rows = lambda t, lo, hi: _out(t, layout, True)[0, lo:hi]
    assert torch.equal(rows(y, 0, 60), rows(y2, 0, 60)) and all(torch.equal(r[n], r2[n]) for n in r)
    x2[0, 28] = float("nan")                               # the last step of the second sequence
    y3, r3 = run(x2, dy)
    assert torch.equal(rows(y, 0, 28), rows(y3, 0, 28)) and torch.equal(rows(y, 29, 60), rows(y3, 29, 60))
    assert torch.equal(rows(r["dx"], 0, 25), rows(r3["dx"], 0, 25)) and torch.equal(rows(r["dx"], 29, 60), rows(r3["dx"], 29, 60))
    assert bool(torch.isnan(rows(y3, 28, 29)).all()) and bool(torch.isnan(rows(r3["dx"], 25, 29)).all())


@pytest.mark.parametrize("io", TYPES)
@pytest.mark.parametrize("layout", LAYOUTS)
def test_reproducible_on_another_stream_and_in_a_graph(api, layout, io):
    import torch
    a, dy, dl = _make(3, layout, 2, 300, 136, 4, io)
    x, dy, w, b, x0, dl = _in(a["x"], layout, False), _in(dy, layout, False), a["weight"].cuda(), a["bias"].cuda(), a["x0"].cuda(), dl.cuda()
    state = x0.clone()

    def run():
        y, last = api.lrnnx_short_conv_fwd(x, w, bias=b, x0=x0, layout=layout, return_last_state=True)
        r = api.lrnnx_short_conv_bwd(x, w, dy, bias=b, x0=x0, dx_last=dl, want_dx0=True, layout=layout)
        return [y, last, *r.values(), api.lrnnx_short_conv_step(last[:, 0], w, state, bias=b), state.clone()]
    first = run()
    state.copy_(x0)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        again = run()
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(first, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for i in range(3):
        x.copy_(torch.randn(x.shape, device="cuda"))
        state.copy_(x0)
        want = [t.clone() for t in run()]
        state.copy_(x0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want)), i


def test_in_place_is_refused(api):
    import torch
    x, dy, w = torch.zeros(2, 9, 8, device="cuda"), torch.zeros(2, 9, 8, device="cuda"), torch.zeros(8, 3, device="cuda")
    with pytest.raises(ValueError):
        api.lrnnx_short_conv_fwd(x, w, out=x)
    for out in (x, dy):
        with pytest.raises(ValueError):
            api.lrnnx_short_conv_bwd(x, w, dy, out=out)
    cu = torch.tensor([0, 9], device="cuda")
    with pytest.raises(ValueError):
        api.lrnnx_short_conv_fwd(x[0], w, cu_seqlens=cu, out=x[0])
