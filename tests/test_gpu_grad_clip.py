"""GPU tests of the norm and the clipping of many tensors against 64 bits.

Tolerances: the norm is rounded once, 6e-8 (held to 1e-7); the scale has a sum, a division and a product, each element one product more: 4 * 6e-8 = 2.4e-7 of every
element, rounded to bfloat16 2^-8."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    import torch
    assert torch.cuda.is_available()
    from paper_2602_08810_amd import api as _api
    _api.lib()
    return _api


def _make(seed, sizes, types="mixed"):
    import torch
    g = torch.Generator().manual_seed(seed)
    pick = {"mixed": lambda i: (torch.float32, torch.bfloat16)[i % 2], "f32": lambda i: torch.float32, "bf16": lambda i: torch.bfloat16}[types]
    return [torch.randn(n, generator=g).mul_(1 + i % 5).to(pick(i)).cuda() for i, n in enumerate(sizes)]


def _norm(grads):
    return math.sqrt(math.fsum(float(t.double().square().sum()) for t in grads))


def _clipped(grads, max_norm):
    scale = min(1.0, max_norm / (_norm(grads) + 1e-6))
    return [t.double() * scale for t in grads]


def _close(got, want):
    import torch
    for a, b in zip(got, want):
        tol = 2.0 ** -8 + 1e-6 if a.dtype == torch.bfloat16 else 2.4e-7
        assert a.shape == b.shape and bool(((a.double() - b).abs() <= tol * b.abs() + 1e-42).all())


@pytest.mark.parametrize("types", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("sizes", [[1], [0, 3], [7, 8, 9, 2048, 8191, 8192, 8193], [100003], [5] * 129, [17, 0, 40000] * 100, [20_000_001, 3]])
def test_norm_and_clip(api, types, sizes):
    import torch
    grads = _make(sum(sizes), sizes, types)
    norm = api.lrnnx_grad_norm(grads)
    want = _norm(grads)
    assert norm.shape == () and abs(norm.item() - want) <= 1e-7 * want
    for max_norm in (0.3 * want, 2 * want + 1):
        ref = _clipped(grads, max_norm)
        out = [torch.full_like(t, 5.0) for t in grads]
        assert api.lrnnx_grad_clip(grads, norm, max_norm, out=out)[0].data_ptr() == out[0].data_ptr()
        _close(out, ref)
        wide = [torch.full(t.shape, 5.0, device="cuda") for t in grads]
        api.lrnnx_grad_clip(grads, norm, max_norm, out=wide)
        _close(wide, ref)
        mine = [t.clone() for t in grads]
        assert all(a is b for a, b in zip(api.lrnnx_grad_clip(mine, norm, max_norm), mine))
        assert all(torch.equal(a, b) for a, b in zip(mine, out))
    assert all(torch.equal(a, b) for a, b in zip(mine, grads))              # below the largest norm: untouched


def test_squares_that_float32_cannot_hold(api):
    import torch
    for value in (1e-30, 3e25, 1e-44):
        t = torch.full((1000,), value, device="cuda")
        want = math.sqrt(1000) * float(t[0].double())
        assert abs(api.lrnnx_grad_norm([t]).item() - want) <= 2e-7 * want + 1e-45
    assert api.lrnnx_grad_norm([torch.full((100,), 3e38, device="cuda")]).item() == float("inf")
    zero = torch.zeros(10, device="cuda")
    assert api.lrnnx_grad_norm([zero]).item() == 0 and not bool(api.lrnnx_grad_clip([zero], api.lrnnx_grad_norm([zero]), 1.0)[0].any())


def test_what_is_not_finite(api):
    import torch
    for bad, rest in ((float("nan"), float("nan")), (float("inf"), 0.0)):
        grads = [torch.ones(50, device="cuda"), torch.ones(20000, dtype=torch.bfloat16, device="cuda")]
        grads[1][777] = bad
        norm = api.lrnnx_grad_norm(grads)
        assert str(norm.item()) == str(bad)
        api.lrnnx_grad_clip(grads, norm, 1.0)
        assert math.isnan(grads[1][777].item()) and str(grads[0][3].item()) == str(rest)


def test_views_that_start_anywhere(api):
    import torch
    flat = torch.randn(70000, device="cuda").to(torch.bfloat16)
    whole = flat.clone()
    parts = [flat[3:20001], flat[20001:20002], flat[20003:69990]]
    want = _clipped(parts, 1.0)
    api.lrnnx_grad_clip(parts, api.lrnnx_grad_norm(parts), 1.0)
    _close(parts, want)
    for i in (0, 1, 2, 20002, 69990, 69999):
        assert flat[i] == whole[i]


def test_reproducible_on_another_stream_and_in_a_graph(api):
    import torch
    grads = _make(1, [30, 40001, 129, 5000] * 50)
    out = [torch.empty_like(t) for t in grads]

    def run():
        norm = api.lrnnx_grad_norm(grads)
        api.lrnnx_grad_clip(grads, norm, 1.0, out=out)
        return [norm] + out
    first = [t.clone() for t in run()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        again = [t.clone() for t in run()]
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(first, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for i in range(3):
        for t in grads:
            t.copy_(torch.randn(t.shape, device="cuda"))
        want = [t.clone() for t in run()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want)), i


def test_results_in_the_place_of_other_gradients_are_refused(api):
    """A result may lie where its own gradient does, and nowhere else among what the call reads or writes."""
    import torch
    room = torch.ones(64, device="cuda")
    g, norm = [room[:8], room[8:16], torch.ones(8, device="cuda").bfloat16()], torch.full((), 2.0, device="cuda")
    fresh = [torch.empty(8, device="cuda") for _ in range(3)]
    wide = torch.ones(16, device="cuda").bfloat16()
    for grads, out in [(g, [g[1], g[0], fresh[0]]), (g, [room[4:12], fresh[1], fresh[2]]), (g, [fresh[0], room[:8], fresh[1]]), (g, [fresh[0], fresh[0], fresh[1]]),
                       (g[:2], [fresh[0], room[12:20]]), ([wide[:8]], [wide.view(torch.float32)])]:
        with pytest.raises(ValueError):
            api.lrnnx_grad_clip(grads, norm, 1.0, out=out)
        with pytest.raises(ValueError):
            api.lrnnx_grad_clip.__wrapped__(grads, norm, 1.0, out=out)
    assert bool((room == 1).all())
    api.lrnnx_grad_clip(g, norm, 1.0, 0.0, out=[g[0], fresh[1], fresh[2]])
    assert bool((g[0] == 0.5).all()) and bool((g[1] == 1).all()) and bool((fresh[1] == 0.5).all()) and bool((fresh[2] == 0.5).all())
    again = [room[8:16], room[8:16]]                       # read twice, written apart
    api.lrnnx_grad_clip(again, norm, 1.0, 0.0, out=fresh[:2])
    assert bool((fresh[0] == 0.5).all()) and bool((fresh[1] == 0.5).all()) and bool((g[1] == 1).all())
