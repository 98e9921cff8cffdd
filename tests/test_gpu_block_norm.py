"""GPU tests of the norms around a block against a plain implementation in 64 bits on the same (rounded) inputs.

Tolerances, of the 2-norm of each tensor: float32 sums over up to 8192 elements or 300 rows, added like independent errors, times the few operations
of a result: 6e-8 * sqrt(300) * 2 = 2e-6, held to 5e-6; results rounded to bfloat16 1.7e-3, held to 4e-3."""
import numpy as np
import pytest

from _delta_ref import norm_bwd, norm_fwd
from _util import rel_l2

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    import torch
    assert torch.cuda.is_available()
    from paper_2602_08810_amd import api as _api
    _api.lib()
    return _api


def _h(t):
    return None if t is None else t.double().cpu().numpy()


def _make(seed, M, D, io, post="full", groups=1, gate=None, residual="f32", scale=True, pre=True):
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    rnd = lambda *s: torch.randn(s, generator=g)
    rt = {"f32": torch.float32, "io": dt, None: dt}[residual]
    a = dict(x=rnd(M, D).to(dt), groups=groups,
             post_weight=1 + 0.3 * rnd(D // groups if post == "shared" else D) if post else None,
             gate=2 * rnd(M, D).to(dt) if gate else None, residual=2 * rnd(M, D).to(rt) if residual else None,
             res_scale=rnd(D) if scale else None, pre_weight=1 + 0.3 * rnd(D) if pre else None)
    a = {n: v.cuda() if torch.is_tensor(v) else v for n, v in a.items()}
    if gate:
        a["gate_act"] = gate
    return a, rnd(M, D).to(rt).cuda(), rnd(M, D).to(dt).cuda() if pre else None


def _ref_args(a):
    return dict(post=_h(a["post_weight"]), groups=a["groups"], gate=_h(a["gate"]), act=a.get("gate_act", "silu"), residual=_h(a["residual"]),
                scale=_h(a["res_scale"]), pre=_h(a["pre_weight"]))


def _check(got, ref, name):
    import torch
    tol = 4e-3 if got.dtype == torch.bfloat16 else 5e-6
    e = rel_l2(_h(got), ref)
    assert e <= tol, f"{name}: relative error {e:.2e}, tolerance {tol:g}"


FORMS = [
    dict(), dict(gate="silu"), dict(gate="sigmoid", residual=None), dict(post=None, gate=None), dict(post=None, gate="silu", scale=False, pre=False),
    dict(scale=False), dict(pre=False), dict(residual=None, scale=False, pre=False, gate="silu"), dict(post=None, residual=None, scale=False),
    dict(residual="io", gate="silu"),
]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("M,D", [(1, 1), (3, 7), (5, 64), (2, 200), (300, 96), (4, 771), (7, 2560), (2, 4100), (2, 8192), (1, 8191)])
def test_widths(api, io, M, D):
    a, dh, dy = _make(M + D, M, D, io, gate="silu")
    _both(api, a, dh, dy)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("form", range(len(FORMS)))
def test_forms(api, io, form):
    a, dh, dy = _make(form, 9, 320, io, **FORMS[form])
    _both(api, a, dh, dy)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("post", ["full", "shared"])
@pytest.mark.parametrize("D,groups", [(64, 64), (96, 2), (96, 12), (2048, 16), (771, 3), (1536, 8), (2560, 4), (4096, 2), (8192, 1024), (90, 9)])
def test_groups(api, io, post, D, groups):
    a, dh, dy = _make(D, 5, D, io, post=post, groups=groups, gate="silu")
    _both(api, a, dh, dy)


def _both(api, a, dh, dy):
    h, y = api.lrnnx_block_norm_fwd(**a)
    ref = _ref_args(a)
    rh, ry, _ = norm_fwd(_h(a["x"]), **ref)
    assert h.dtype == (a["residual"] if a["residual"] is not None else a["x"]).dtype
    _check(h, rh, "h")
    assert (y is None) == (ry is None)
    if y is not None:
        _check(y, ry, "y")
    r = api.lrnnx_block_norm_bwd(dh=dh, dy=dy, **a)
    want = norm_bwd(_h(dh), _h(dy), _h(a["x"]), **ref)
    assert set(r) == set(want)
    for n in want:
        _check(r[n], want[n], n)


def test_strided_rows_and_only_one_gradient(api):
    import torch
    a, dh, dy = _make(1, 12, 136, "bf16", gate="silu")
    wide = torch.zeros(12, 512, dtype=torch.bfloat16, device="cuda")
    wide[:, 3:139], wide[:, 200:336] = a["x"], a["gate"]
    views = {**a, "x": wide[:, 3:139], "gate": wide[:, 200:336]}
    for x, y in zip(api.lrnnx_block_norm_fwd(**views), api.lrnnx_block_norm_fwd(**a)):
        assert rel_l2(_h(x), _h(y)) <= 4e-3
    for kw in (dict(dh=dh), dict(dy=dy)):
        r = api.lrnnx_block_norm_bwd(**kw, **views)
        want = norm_bwd(_h(kw.get("dh")), _h(kw.get("dy")), _h(a["x"]), **_ref_args(a))
        for n in want:
            if np.abs(want[n]).max() > 0:
                _check(r[n], want[n], n)
            else:
                assert not bool(r[n].any())
    h3, y3 = api.lrnnx_block_norm_fwd(**{**a, **{n: a[n].view(3, 4, 136) for n in ("x", "gate", "residual")}})
    h, y = api.lrnnx_block_norm_fwd(**a)
    assert torch.equal(h3.view(12, 136), h) and torch.equal(y3.view(12, 136), y)


def test_residual_in_place_zero_rows_and_infinities(api):
    import torch
    a, dh, dy = _make(2, 6, 256, "f32")
    a["x"][2], a["residual"][2] = 0, 0                       # a row of zeros: rms is sqrt(eps)
    want = api.lrnnx_block_norm_fwd(**a)
    keep = a["residual"].clone()
    h, y = api.lrnnx_block_norm_fwd(**a, out=a["residual"])
    assert h.data_ptr() == a["residual"].data_ptr() and torch.equal(h, want[0]) and torch.equal(y, want[1])
    assert not bool(y[2].any())
    a["residual"] = keep
    r = api.lrnnx_block_norm_bwd(dh=dh, dy=dy, **a)
    assert all(bool(torch.isfinite(v).all()) for v in r.values())
    a["residual"][4, 5] = float("inf")                       # one row is lost, no other
    h, y = api.lrnnx_block_norm_fwd(**a)
    rows = [0, 1, 2, 3, 5]
    assert torch.equal(h[rows], want[0][rows]) and torch.equal(y[rows], want[1][rows]) and bool(torch.isnan(y[4]).any())


def test_reproducible_and_in_a_graph(api):
    import torch
    a, dh, dy = _make(3, 3000, 512, "bf16", gate="silu", groups=4, post="shared")
    first = api.lrnnx_block_norm_bwd(dh=dh, dy=dy, **a)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        again = api.lrnnx_block_norm_bwd(dh=dh, dy=dy, **a)
    side.synchronize()
    assert all(torch.equal(first[n], again[n]) for n in first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h, y = api.lrnnx_block_norm_fwd(**a)
        r = api.lrnnx_block_norm_bwd(dh=dh, dy=dy, **a)
    for i in range(3):
        a["x"].copy_(torch.randn(a["x"].shape, device="cuda"))
        wh, wy = api.lrnnx_block_norm_fwd(**a)
        want = api.lrnnx_block_norm_bwd(dh=dh, dy=dy, **a)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(h, wh) and torch.equal(y, wy) and all(torch.equal(r[n], want[n]) for n in r), i


def test_refusals(api):
    import torch
    a, dh, dy = _make(4, 4, 96, "bf16", gate="silu")
    bad = [
        (dict(groups=5), ValueError), (dict(post_weight=a["post_weight"].bfloat16()), TypeError), (dict(pre_weight=a["pre_weight"][:95]), ValueError),
        (dict(gate=a["gate"].float()), TypeError), (dict(gate=a["gate"][:3]), ValueError), (dict(residual=a["residual"].double()), TypeError),
        (dict(gate_act="relu"), KeyError), (dict(x=a["x"].cpu()), TypeError), (dict(x=a["x"].half()), TypeError),
        (dict(x=a["x"].t().contiguous().t()), ValueError), (dict(out=torch.empty(4, 97, device="cuda")), (TypeError, ValueError)),
    ]
    for change, error in bad:
        with pytest.raises(error):
            api.lrnnx_block_norm_fwd(**{**a, **change})
    with pytest.raises(ValueError):
        api.lrnnx_block_norm_bwd(**a)
    with pytest.raises(api.LrnnxError) as e:
        api.lrnnx_block_norm_fwd(torch.zeros(1, 8200, device="cuda"), pre_weight=torch.ones(8200, device="cuda"))
    assert e.value.code == 2
    with pytest.raises(api.LrnnxError) as e:
        api.lrnnx_block_norm_bwd(dh=dh, dy=dy, **a, workspace=torch.empty(32, dtype=torch.uint8, device="cuda"))
    assert e.value.code == 3


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("M,D,groups", [(3, 2731, 1), (600, 4097, 1), (2, 5001, 1), (700, 6145, 5), (300, 8190, 3), (520, 8191, 1), (1100, 288, 32),
                                        (600, 1568, 32), (257, 1026, 2)])
def test_widths_that_nothing_divides(api, io, M, D, groups):
    """Rows that are read an element at a time, several rows a workgroup, and groups that are neither the row nor a power of two of its pieces."""
    a, dh, dy = _make(M + D, M, D, io, groups=groups, gate="sigmoid")
    _both(api, a, dh, dy)
