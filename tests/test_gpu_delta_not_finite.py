"""Numbers that are not finite in the gated delta rule, forward: a step's are seen by that step and later ones, of its head (of v: its column), and by
nothing before.  Equal bits everywhere else: what is finite goes through the same arithmetic."""
import pytest

from test_gpu_gated_delta import _make, _state, api  # noqa: F401

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
FORMS = [  # B, L, Hk, Hv, dk, dv: few heads, many, in segments, odd widths, shared heads
    (1, 100, 2, 2, 64, 64), (2, 70, 70, 70, 128, 64), (1, 1100, 1, 1, 128, 96), (2, 75, 1, 2, 44, 33), (1, 70, 24, 72, 64, 40),
]


def _run(api, t, s0, save):  # noqa: F811
    o, last, *_ = api.lrnnx_gated_delta_fwd(**t, s0=s0, return_last_state=True, return_saved=save)
    return o, last


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("save", [False, True])
@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("what", [INF, -INF, NAN])
def test_values(api, io, save, form, what):  # noqa: F811
    import torch
    B, L, Hk, Hv, dk, dv = FORMS[form]
    t, s0 = _make(1, (B, L), Hk, Hv, dk, dv, io), _state(2, B, Hv, dk, dv)
    clean, clean_last = _run(api, t, s0, save)
    for at in (0, 9, 31, 32, 47, L - 1):
        bad = dict(t, v=t["v"].clone())
        c, h, b = (5 * at) % dv, Hv - 1, B - 1
        bad["v"][b, at, h, c] = what
        o, last = _run(api, bad, s0, save)
        same = torch.ones_like(clean, dtype=torch.bool)
        same[b, at:, h, c] = False
        assert torch.equal(o[same], clean[same]), at
        assert not bool(torch.isfinite(o[~same]).any()), at
        same = torch.ones_like(last, dtype=torch.bool)
        same[b, h, :, c] = False
        assert torch.equal(last[same], clean_last[same]) and not bool(torch.isfinite(last[~same]).any()), at


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("save", [False, True])
@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("name,what", [("k", INF), ("k", NAN), ("beta", NAN), ("beta", INF), ("g", NAN), ("g", INF)])
def test_keys_and_gates(api, io, save, form, name, what):  # noqa: F811
    import torch
    B, L, Hk, Hv, dk, dv = FORMS[form]
    t, s0 = _make(3, (B, L), Hk, Hv, dk, dv, io), _state(4, B, Hv, dk, dv)
    clean, clean_last = _run(api, t, s0, save)
    for at in (0, 9, 31, 32, 47, L - 1):
        bad = {**t, name: t[name].clone()}
        if name == "k":
            bad["k"][0, at, Hk - 1, (3 * at) % dk] = what
            heads = slice(Hv - Hv // Hk, Hv)
        else:
            bad[name][0, at, Hv - 1] = what
            heads = slice(Hv - 1, Hv)
        o, last = _run(api, bad, s0, save)
        same = torch.ones_like(clean, dtype=torch.bool)
        same[0, at:, heads] = False
        assert torch.equal(o[same], clean[same]), at
        assert not bool(torch.isfinite(o[~same]).any()), at
        same = torch.ones_like(last, dtype=torch.bool)
        same[0, heads] = False
        assert torch.equal(last[same], clean_last[same]) and not bool(torch.isfinite(last[~same]).any()), at


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("what", [INF, NAN])
def test_queries_and_the_first_state(api, io, form, what):  # noqa: F811
    import torch
    B, L, Hk, Hv, dk, dv = FORMS[form]
    t, s0 = _make(5, (B, L), Hk, Hv, dk, dv, io), _state(6, B, Hv, dk, dv)
    clean, clean_last = _run(api, t, s0, False)
    for at in (0, 31, 40, L - 1):                                # a query reads and leaves nothing behind
        bad = dict(t, q=t["q"].clone())
        bad["q"][0, at, 0, dk // 2] = what
        o, last = _run(api, bad, s0, False)
        same = torch.ones_like(clean, dtype=torch.bool)
        same[0, at, :Hv // Hk] = False
        assert torch.equal(o[same], clean[same]) and torch.equal(last, clean_last), at
        assert not bool(torch.isfinite(o[~same]).any()), at
    first = s0.clone()
    first[0, 0, dk // 3, dv // 2] = what
    o, last = _run(api, t, first, False)
    same = torch.ones_like(clean, dtype=torch.bool)
    same[0, :, 0, dv // 2] = False
    assert torch.equal(o[same], clean[same]) and not bool(torch.isfinite(o[~same]).any())
    same = torch.ones_like(last, dtype=torch.bool)
    same[0, 0, :, dv // 2] = False
    assert torch.equal(last[same], clean_last[same]) and not bool(torch.isfinite(last[~same]).any())


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_what_is_saved_of_earlier_steps(api, io):  # noqa: F811
    """dq of the steps before one in v that is not finite, and all of dv, which does not depend on v."""
    import torch
    t, do = _make(7, (1, 128), 2, 2, 64, 64, io, "io"), _make(8, (1, 128), 2, 2, 64, 64, io)["v"]

    def grads(v):
        _, saved = api.lrnnx_gated_delta_fwd(**dict(t, v=v), return_saved=True)
        return api.lrnnx_gated_delta_bwd(**dict(t, v=v), do=do, saved=saved)

    for at in (3, 45, 70):
        bad = t["v"].clone()
        bad[0, at, 1, 20] = NAN
        a, b = grads(t["v"]), grads(bad)
        assert torch.equal(a["dv"], b["dv"])
        assert torch.equal(a["dq"][:, :at], b["dq"][:, :at]) and torch.equal(a["dq"][:, :, 0], b["dq"][:, :, 0])
        assert torch.equal(a["dk"][:, :at], b["dk"][:, :at])
        assert not bool(torch.isfinite(b["dq"][0, at:, 1]).any())


@pytest.mark.parametrize("io,gates,states", [("bf16", "io", False), ("bf16", "io", True), ("bf16", None, True), ("f32", None, True), ("f32", None, False)])
@pytest.mark.parametrize("save", [False, True])
@pytest.mark.parametrize("B,L,Hk,Hv,dk,dv", [(2, 70, 70, 70, 64, 64), (2, 70, 70, 70, 128, 64), (1, 100, 2, 2, 64, 64), (1, 100, 2, 2, 128, 48), (1, 1100, 1, 1, 64, 96),
                                            (1, 2570, 24, 24, 16, 64)])
def test_every_form_of_the_walk(api, io, gates, states, save, B, L, Hk, Hv, dk, dv):  # noqa: F811
    """With and without states (bfloat16 gates then take two planes), one wavefront to 16 columns or two, in segments of either."""
    import torch
    t, s0 = _make(9, (B, L), Hk, Hv, dk, dv, io, gates), _state(10, B, Hv, dk, dv) if states else None

    def run(t):
        r = api.lrnnx_gated_delta_fwd(**t, s0=s0, return_last_state=states, return_saved=save)
        return r[0] if isinstance(r, tuple) else r

    clean = run(t)
    for at in (0, 20, 31, 50, L - 1):
        for name, what in (("v", NAN), ("v", INF), ("k", NAN), ("beta", INF), ("g", NAN)):
            bad = {**t, name: t[name].clone()}
            same = torch.ones_like(clean, dtype=torch.bool)
            if name == "v":
                bad["v"][0, at, Hv - 1, dv // 2] = what
                same[0, at:, Hv - 1, dv // 2] = False
            elif name == "k":
                bad["k"][0, at, Hk - 1, dk - 1] = what
                same[0, at:, Hv - Hv // Hk:] = False
            else:
                bad[name][0, at, Hv - 1] = what
                same[0, at:, Hv - 1] = False
            o = run(bad)
            assert torch.equal(o[same], clean[same]), (name, what, at)
            assert not bool(torch.isfinite(o[~same]).any()), (name, what, at)
