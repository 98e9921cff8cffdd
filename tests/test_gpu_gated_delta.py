"""GPU tests of the gated delta rule against a plain implementation in 64 bits on the same (rounded) inputs.

Tolerances, of the 2-norm of each tensor.  float32: products and sums are float32 (unit roundoff 6e-8); errors of a step live as long as
the memory, at most some hundred steps here, and add up like independent ones, 6e-8 * sqrt(1000) * 10 for the handful of products a result goes
through: 2e-5.  bfloat16: rounding a result costs 2^-9 at most, 1.7e-3 in the norm; the gradients take the saved states, rounded once, as
factors (twice: S0 and dS1), so sqrt(3) * 1.7e-3 in all, held to 6e-3.  Gradients of float32 gates with bfloat16 I/O: the states' rounding
alone, in sums that cancel: 1e-2."""
import numpy as np
import pytest

from _delta_ref import delta_bwd, delta_fwd
from _util import rel_l2

pytestmark = pytest.mark.gpu
F32, BF16 = 2e-5, 6e-3


@pytest.fixture(scope="module")
def api():
    import torch
    assert torch.cuda.is_available()
    from paper_2602_08810_amd import api as _api
    _api.lib()
    return _api


def _t(x, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(dtype).cuda()


def _h(t):
    return t.double().cpu().numpy()


def _make(seed, lead, Hk, Hv, dk, dv, io, gates=None, state=True, rate=0.3, views=False):
    """Device tensors (leading axes `lead`); io "f32" or "bf16"."""
    import torch
    rng = np.random.default_rng(seed)
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    gt = dt if gates == "io" else torch.float32
    unit = lambda x: x / np.linalg.norm(x, axis=-1, keepdims=True)
    q, k, v = unit(rng.normal(size=(*lead, Hk, dk))), unit(rng.normal(size=(*lead, Hk, dk))), rng.normal(size=(*lead, Hv, dv))
    t = dict(q=_t(q, dt), k=_t(k, dt), v=_t(v, dt), g=_t(-rate * rng.exponential(size=(*lead, Hv)), gt),
             beta=_t(rng.uniform(0, 1, (*lead, Hv)), gt))
    if views:                                # slices of one buffer whose rows start at odd places
        fused = torch.zeros((*lead, 2 * Hk * dk + Hv * dv + 3), dtype=dt, device="cuda")
        at = 1
        for n, H, d in (("q", Hk, dk), ("k", Hk, dk), ("v", Hv, dv)):
            view = fused[..., at:at + H * d].unflatten(-1, (H, d))
            view.copy_(t[n])
            t[n] = view
            at += H * d
        t["g"] = t["g"].transpose(-1, -2).contiguous().transpose(-1, -2)
    return t


def _state(seed, n, Hv, dk, dv):
    return _t(0.5 * np.random.default_rng(seed).normal(size=(n, Hv, dk, dv)), __import__("torch").float32)


def _reference(t, scale, s0=None, do=None, ds_last=None, spans=None):
    """Stacked reference results of every sequence: entries of the batch, or `spans` of a packed axis."""
    a = {n: _h(x) for n, x in t.items()}
    rows = [slice(lo, hi) for lo, hi in spans] if spans is not None else range(a["v"].shape[0])
    fwd, bwd = [], []
    for i, r in enumerate(rows):
        one = [a[n][r] for n in ("q", "k", "v", "g", "beta")]
        s = None if s0 is None else _h(s0[i])
        o, states, _ = delta_fwd(*one, scale, s)
        fwd.append((o, states[-1]))
        if do is not None:
            bwd.append(delta_bwd(*one, scale, _h(do)[r], s, None if ds_last is None else _h(ds_last[i])))
    return fwd, bwd


def _near(got, ref, tol, where):
    e = rel_l2(_h(got), ref)
    assert e <= tol, f"{where}: relative error {e:.2e}, tolerance {tol:g}"


SHAPES = [  # L, Hk, Hv, dk, dv
    (1, 1, 1, 1, 1), (2, 1, 2, 3, 5), (31, 2, 2, 8, 16), (32, 1, 1, 64, 64), (33, 2, 4, 44, 76), (63, 1, 3, 65, 33),
    (64, 1, 1, 128, 128), (65, 2, 2, 128, 128), (100, 1, 2, 96, 80), (130, 1, 1, 128, 256), (257, 2, 2, 64, 31),
]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("L,Hk,Hv,dk,dv", SHAPES)
def test_forward_and_backward(api, io, L, Hk, Hv, dk, dv):
    B, scale = 2, dk ** -0.5
    t = _make(L + dk, (B, L), Hk, Hv, dk, dv, io, gates="io", views=L % 2 == 1)
    s0, dl = _state(1, B, Hv, dk, dv), _state(2, B, Hv, dk, dv)
    do = _make(9, (B, L), Hk, Hv, dk, dv, io)["v"]
    o, last, saved = api.lrnnx_gated_delta_fwd(**t, s0=s0, return_last_state=True, return_saved=True)
    r = api.lrnnx_gated_delta_bwd(**t, do=do, saved=saved, s0=s0, ds_last=dl, want_ds0=True)
    fwd, bwd = _reference(t, scale, s0, do, dl)
    tol = F32 if io == "f32" else BF16
    _near(o, np.stack([f[0] for f in fwd]), tol, "o")
    _near(last, np.stack([f[1] for f in fwd]), F32, "last state")
    for n in ("dq", "dk", "dv", "dg", "dbeta"):
        _near(r[n], np.stack([b[n] for b in bwd]), tol, n)
    _near(r["ds0"], np.stack([b["ds0"] for b in bwd]), F32, "ds0")


@pytest.mark.parametrize("io,gates", [("f32", None), ("bf16", None), ("bf16", "io")])
def test_without_states(api, io, gates):
    """No first state, no last one wanted: the shorter arithmetic of results in bfloat16; gates in float32 or in the I/O type."""
    B, L, Hk, Hv, dk, dv = 3, 150, 2, 4, 128, 64
    t = _make(5, (B, L), Hk, Hv, dk, dv, io, gates, rate=0.05)
    do = _make(6, (B, L), Hk, Hv, dk, dv, io)["v"]
    o, saved = api.lrnnx_gated_delta_fwd(**t, return_saved=True, scale=0.3)
    alone = api.lrnnx_gated_delta_fwd(**t, scale=0.3)
    assert __import__("torch").equal(o, alone)
    r = api.lrnnx_gated_delta_bwd(**t, do=do, saved=saved, scale=0.3)
    assert set(r) == {"dq", "dk", "dv", "dg", "dbeta"}
    fwd, bwd = _reference(t, 0.3, None, do)
    tol = F32 if io == "f32" else BF16
    _near(o, np.stack([f[0] for f in fwd]), tol, "o")
    for n in r:
        loose = io == "bf16" and gates is None and n in ("dg", "dbeta")
        assert r[n].dtype == t[n[1:]].dtype
        _near(r[n], np.stack([b[n] for b in bwd]), 1e-2 if loose else tol, n)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 96), (40, 24)])
def test_packed(api, io, dk, dv):
    """Sequences of 0 to 200 steps that start anywhere; what lies outside them is NaN and stays outside."""
    import torch
    lens, L, Hk, Hv = [5, 0, 1, 64, 63, 0, 130, 32, 200, 0], 520, 2, 4
    cu = np.concatenate([[7], 7 + np.cumsum(lens)])
    spans = list(zip(cu[:-1], cu[1:]))
    t = _make(11, (L,), Hk, Hv, dk, dv, io)
    for x in t.values():
        x[:7] = float("nan")
        x[cu[-1]:] = float("nan")
    s0, dl = _state(3, len(lens), Hv, dk, dv), _state(4, len(lens), Hv, dk, dv)
    do = _make(12, (L,), Hk, Hv, dk, dv, io)["v"]
    do[:7] = float("nan")
    cut = torch.tensor(cu, dtype=torch.int64, device="cuda")
    out = torch.full((L, Hv, dv), 7.0, dtype=do.dtype, device="cuda")
    o, last, saved = api.lrnnx_gated_delta_fwd(**t, s0=s0, cu_seqlens=cut, return_last_state=True, return_saved=True, out=out)
    r = api.lrnnx_gated_delta_bwd(**t, do=do, saved=saved, s0=s0, ds_last=dl, want_ds0=True, cu_seqlens=cut)
    fwd, bwd = _reference(t, dk ** -0.5, s0, do, dl, spans)
    tol = F32 if io == "f32" else BF16
    inside = slice(7, cu[-1])
    assert bool((out[:7] == 7).all()) and bool((out[cu[-1]:] == 7).all())
    _near(o[inside], np.concatenate([f[0] for f in fwd]), tol, "o")
    _near(last, np.stack([f[1] for f in fwd]), F32, "last state")
    for n in ("dq", "dk", "dv", "dg", "dbeta"):
        loose = io == "bf16" and n in ("dg", "dbeta")
        _near(r[n][inside], np.concatenate([b[n] for b in bwd]), 1e-2 if loose else tol, n)
    _near(r["ds0"], np.stack([b["ds0"] for b in bwd]), F32, "ds0")
    empty = [i for i, n in enumerate(lens) if n == 0]
    assert torch.equal(last[empty], s0[empty]) and torch.equal(r["ds0"][empty], dl[empty])


def test_a_sequence_does_not_see_its_neighbours_nan(api):
    import torch
    t = _make(21, (200,), 1, 1, 64, 64, "bf16")
    cut = torch.tensor([0, 70, 130, 200], dtype=torch.int64, device="cuda")
    do = _make(22, (200,), 1, 1, 64, 64, "bf16")["v"]
    clean, saved = api.lrnnx_gated_delta_fwd(**t, cu_seqlens=cut, return_saved=True)
    rc = api.lrnnx_gated_delta_bwd(**t, do=do, saved=saved, cu_seqlens=cut)
    for x in (*t.values(), do):
        x[70:130] = float("nan")
    o, saved = api.lrnnx_gated_delta_fwd(**t, cu_seqlens=cut, return_saved=True)
    r = api.lrnnx_gated_delta_bwd(**t, do=do, saved=saved, cu_seqlens=cut)
    for a, b in [(o, clean)] + [(r[n], rc[n]) for n in r]:
        assert torch.equal(a[:70], b[:70]) and torch.equal(a[130:], b[130:])
        assert bool(torch.isnan(a[70:130]).any())


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["forget", "keep", "strong", "beta0", "same_keys", "beta2"])
def test_gates_at_their_ends(api, io, kind):
    """Steps that forget everything (g = -inf), decays of 1 and of e^-60 a step, beta 0, one key written again and again with beta 1 (the
    solve is then as far from the identity as it gets), beta 2."""
    B, L, H, dk, dv = 1, 140, 2, 32, 32
    t = _make(31, (B, L), H, H, dk, dv, io, rate=0.2)
    if kind == "forget":
        t["g"][:, [0, 40, 41, 64, 100]] = float("-inf")
    if kind == "keep":
        t["g"].zero_()
    if kind == "strong":
        t["g"].fill_(-60.0)
        t["g"][:, ::3] = -1e-3
    if kind == "beta0":
        t["beta"][:, 20:90] = 0
    if kind == "same_keys":
        t["k"].copy_(t["k"][:, :1].expand_as(t["k"]))
        t["beta"].fill_(1.0)
        t["g"].fill_(-1e-3)
    if kind == "beta2":
        t["beta"].fill_(1.9)
    s0, dl = _state(7, B, H, dk, dv), _state(8, B, H, dk, dv)
    do = _make(32, (B, L), H, H, dk, dv, io)["v"]
    o, last, saved = api.lrnnx_gated_delta_fwd(**t, s0=s0, return_last_state=True, return_saved=True)
    r = api.lrnnx_gated_delta_bwd(**t, do=do, saved=saved, s0=s0, ds_last=dl, want_ds0=True)
    fwd, bwd = _reference(t, dk ** -0.5, s0, do, dl)
    tol = F32 if io == "f32" else BF16
    _near(o[0], fwd[0][0], tol, "o")
    _near(last[0], fwd[0][1], F32, "last state")
    for n in ("dq", "dk", "dv", "dg", "dbeta"):
        loose = io == "bf16" and n in ("dg", "dbeta")
        _near(r[n][0], bwd[0][n], 1e-2 if loose else tol, n)
    _near(r["ds0"][0], bwd[0]["ds0"], F32, "ds0")


def test_gradients_against_differences(api):
    """Directional differences of the forward call itself in float32 (step 1e-2, central: truncation of order 1e-4 of the value, rounding of the
    loss 1e-6 / 1e-2): held to 2e-3 of the largest directional derivative's scale."""
    import torch
    B, L, H, dk, dv = 1, 70, 2, 16, 12
    t = _make(41, (B, L), H, H, dk, dv, "f32")
    s0 = _state(42, B, H, dk, dv)
    do, dl = _make(43, (B, L), H, H, dk, dv, "f32")["v"], _state(44, B, H, dk, dv)
    _, saved = api.lrnnx_gated_delta_fwd(**t, s0=s0, return_saved=True)
    r = api.lrnnx_gated_delta_bwd(**t, do=do, saved=saved, s0=s0, ds_last=dl, want_ds0=True)

    def loss(t, s0):
        o, last = api.lrnnx_gated_delta_fwd(**t, s0=s0, return_last_state=True)
        return float((o.double() * do).sum() + (last.double() * dl).sum())

    gen = torch.Generator(device="cuda").manual_seed(5)
    for n in ("q", "k", "v", "g", "beta", "s0"):
        base = s0 if n == "s0" else t[n]
        d = torch.randn(base.shape, generator=gen, device="cuda")
        d /= d.norm()
        ends = [loss(t, base + e * d) if n == "s0" else loss({**t, n: base + e * d}, s0) for e in (1e-2, -1e-2)]
        want = float((r["ds0" if n == "s0" else "d" + n].double() * d).sum())
        scale = float(r["ds0" if n == "s0" else "d" + n].double().norm()) / np.sqrt(base.numel())
        assert abs((ends[0] - ends[1]) / 2e-2 - want) <= 2e-3 * max(abs(want), scale), n


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("B,Hk,Hv,dk,dv", [(1, 1, 1, 1, 1), (3, 2, 4, 128, 128), (2, 1, 3, 44, 77), (2, 2, 2, 31, 256), (5, 1, 1, 96, 34)])
def test_steps_reproduce_the_sequence(api, io, B, Hk, Hv, dk, dv):
    import torch
    L = 9
    t = _make(51, (B, L), Hk, Hv, dk, dv, io, gates="io" if dk > 64 else None, views=True)
    s0 = _state(52, B, Hv, dk, dv)
    fwd, _ = _reference(t, dk ** -0.5, s0)
    state = s0.clone()
    o = torch.empty((B, L, Hv, dv), dtype=t["v"].dtype, device="cuda")
    for i in range(L):                                       # slices of the sequence's tensors, written into one
        one = {n: x[:, i] for n, x in t.items()}
        y = api.lrnnx_gated_delta_step(**one, state=state, out=o[:, i])
        assert y.data_ptr() == o[:, i].data_ptr()
    tol = F32 if io == "f32" else BF16
    _near(o, np.stack([f[0] for f in fwd]), tol, "o")
    _near(state, np.stack([f[1] for f in fwd]), F32, "state")


def test_step_forgets_and_keeps(api):
    import torch
    t = _make(61, (2, 1), 1, 1, 8, 8, "f32")
    one = {n: x[:, 0] for n, x in t.items()}
    one["g"][0], one["beta"][1] = float("-inf"), 0.0
    state = _state(62, 2, 1, 8, 8)
    before = state.clone()
    o = api.lrnnx_gated_delta_step(**one, state=state)
    assert bool(torch.isfinite(o).all())
    want = one["k"][0, 0][:, None] * (one["beta"][0] * one["v"][0, 0])[None, :]
    assert torch.allclose(state[0, 0], want, atol=1e-6)
    assert torch.allclose(state[1], before[1] * torch.exp(one["g"][1]), atol=1e-6)


def test_results_are_reproducible_on_any_stream(api):
    import torch
    t = _make(71, (2, 300), 2, 4, 128, 128, "bf16", "io")
    do = _make(72, (2, 300), 2, 4, 128, 128, "bf16")["v"]

    def once():
        o, saved = api.lrnnx_gated_delta_fwd(**t, return_saved=True)
        return [o, *api.lrnnx_gated_delta_bwd(**t, do=do, saved=saved).values()]

    first = once()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = once()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_calls_in_a_graph(api):
    """Forward, backward and step captured once and replayed on new inputs, eager work between the replays."""
    import torch
    t = _make(81, (2, 100), 1, 2, 64, 64, "bf16", "io")
    do = _make(82, (2, 100), 1, 2, 64, 64, "bf16")["v"]
    state = _state(83, 2, 2, 64, 64)

    def once():
        o, saved = api.lrnnx_gated_delta_fwd(**t, return_saved=True)
        r = api.lrnnx_gated_delta_bwd(**t, do=do, saved=saved)
        y = api.lrnnx_gated_delta_step(*(t[n][:, 0] for n in ("q", "k", "v", "g", "beta")), state)
        return [o, y, *r.values()]

    once()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    start = state.clone()
    with torch.cuda.graph(graph):
        captured = once()
    for i in range(3):
        fresh = _make(90 + i, (2, 100), 1, 2, 64, 64, "bf16", "io")
        for n in t:
            t[n].copy_(fresh[n])
        state.copy_(start)
        want = [x.clone() for x in once()]
        after = state.clone()
        state.copy_(start)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want)), i
        assert torch.equal(state, after)


def test_offsets_beyond_32_bits(api):
    """Rows 1.3e9 elements apart: the last of three steps starts 2.6e9 elements in."""
    import torch
    far, d = 1_300_000_000, 64
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("not enough memory")
    t = _make(101, (1, 3), 1, 1, d, d, "bf16")
    do = _make(102, (1, 3), 1, 1, d, d, "bf16")["v"]
    want, saved = api.lrnnx_gated_delta_fwd(**t, return_saved=True)
    rw = api.lrnnx_gated_delta_bwd(**t, do=do, saved=saved)
    big = torch.empty(2 * far + 8 * d, dtype=torch.bfloat16, device="cuda")
    views = {}
    for i, n in enumerate(("q", "k", "v")):
        views[n] = big[i * d:].as_strided((1, 3, 1, d), (far, far, d, 1))
        views[n].copy_(t[n])
    out, dov = (big[i * d:].as_strided((1, 3, 1, d), (far, far, d, 1)) for i in (3, 4))
    dov.copy_(do)
    got, saved = api.lrnnx_gated_delta_fwd(**{**t, **views}, out=out, return_saved=True)
    r = api.lrnnx_gated_delta_bwd(**{**t, **views}, do=dov, saved=saved)
    assert torch.equal(got, want) and all(torch.equal(r[n], rw[n]) for n in r)


def test_refusals(api):
    import torch
    t = _make(111, (2, 8), 2, 4, 16, 16, "bf16")
    bad = [
        (dict(q=t["q"].float()), TypeError), (dict(k=t["k"][:, :7]), ValueError), (dict(v=t["v"][:, :, :3]), ValueError),
        (dict(g=t["g"].to(torch.float64)), TypeError), (dict(beta=t["beta"][:, :, :2]), ValueError),
        (dict(g=t["g"].bfloat16()), TypeError), (dict(s0=torch.zeros(2, 4, 16, 8, device="cuda")), ValueError),
        (dict(q=t["q"].transpose(2, 3).contiguous().transpose(2, 3)), ValueError),
        (dict(out=torch.empty(1, device="cuda", dtype=torch.bfloat16).expand(2, 8, 4, 16)), ValueError),
        (dict(v=t["v"].cpu()), TypeError),
    ]
    for change, error in bad:
        with pytest.raises(error):
            api.lrnnx_gated_delta_fwd(**{**t, **change})
    wide = _make(112, (1, 4), 1, 1, 129, 8, "f32")
    with pytest.raises(api.LrnnxError) as e:
        api.lrnnx_gated_delta_fwd(**wide)
    assert e.value.code == 2
    tall = _make(113, (1, 4), 1, 1, 8, 257, "f32")
    with pytest.raises(api.LrnnxError) as e:
        api.lrnnx_gated_delta_fwd(**tall)
    assert e.value.code == 2
    with pytest.raises(api.LrnnxError) as e:
        api.lrnnx_gated_delta_fwd(**t, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.code == 3
    _, saved = api.lrnnx_gated_delta_fwd(**t, return_saved=True)
    with pytest.raises(api.LrnnxError) as e:
        api.lrnnx_gated_delta_bwd(**t, do=t["v"], saved=saved[:1024])
    assert e.value.code == 3
    with pytest.raises(ValueError):
        api.lrnnx_gated_delta_step(*(t[n][:, 0] for n in ("q", "k", "v", "g", "beta")), torch.zeros(2, 4, 16, 17, device="cuda"))
    with pytest.raises(TypeError):
        api.lrnnx_gated_delta_step(*(t[n][:, 0] for n in ("q", "k", "v", "g", "beta")), torch.zeros(2, 4, 16, 16, device="cuda").bfloat16())
