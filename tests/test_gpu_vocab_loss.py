"""GPU tests of the loss over a vocabulary against a plain implementation in 64 bits on the same (rounded) inputs.

Tolerances, of the 2-norm of each tensor.  A logit is a sum of up to 771 products in float32 on the matrix units (32 at a time): 6e-8 * sqrt(771 / 32) of
its terms' size, 3e-7; its exponential is off by as much and by the hardware's 1e-7 (1 + |z|), |z| < 10, their logarithm's sum by less: lse and loss 2e-6.
Gradients in float32: the exponentials' 1.5e-6, sums like the logits': held to 5e-6.  In bfloat16 dz is rounded (rms 1.7e-3 of it, independent errors) and the
result too: 1.7e-3 * sqrt(2) = 2.4e-3, held to 4e-3."""
import pytest

from _train_ref import vocab

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    import torch
    assert torch.cuda.is_available()
    from paper_2602_08810_amd import api as _api
    _api.lib()
    return _api


def _make(seed, T, V, K, io, none=0.3):
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    w = (torch.randn(V, K, generator=g) * 1.5 * K ** -0.5).to(dt)
    target = torch.randint(0, V, (T,), generator=g)
    h = (torch.randn(T, K, generator=g) + 3 * torch.rand(T, 1, generator=g) * w[target].float()).to(dt)
    target[torch.rand(T, generator=g) < none] = -100
    return h, w, target, torch.rand(T, generator=g) + 0.1


def _check(got, want, name, tol=None):
    import torch
    tol = tol or (4e-3 if got.dtype == torch.bfloat16 else 5e-6 if name.startswith("d") else 2e-6)
    got = got.double().cpu()
    assert got.shape == want.shape, name
    e = ((got - want).norm() / want.norm().clamp(min=1e-300)).item()
    assert e <= tol, f"{name}: relative error {e:.2e}, tolerance {tol:g}"


def _both(api, h, w, target, dloss):
    loss, lse = api.lrnnx_vocab_loss_fwd(h.cuda(), w.cuda(), target.cuda())
    r = api.lrnnx_vocab_loss_bwd(h.cuda(), w.cuda(), target.cuda(), lse, dloss.cuda())
    want = vocab(h.double(), w.double(), target, dloss.double())
    for n, got, ref in zip(("loss", "lse", "dh", "dweight"), (loss, lse, r["dh"], r["dweight"]), want):
        _check(got, ref, n)
    return loss, lse, r


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,K", [(1, 1, 1), (1, 300, 64), (3, 5, 7), (5, 256, 8), (17, 257, 72), (64, 1000, 128), (255, 255, 136), (257, 513, 64),
                                   (300, 771, 200), (70, 2000, 771), (600, 300, 330), (33, 3500, 65),
                                   (2500, 130, 40), (4500, 60, 24), (5, 9000, 40), (1, 5000, 300), (700, 2100, 136)])
def test_sizes(api, io, T, V, K):
    _both(api, *_make(T + V + K, T, V, K, io))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("none", [0.0, 1.0, 0.97])
def test_rows_without_a_target(api, io, none):
    h, w, target, dloss = _make(1, 270, 300, 96, io, none)
    loss, lse, r = _both(api, h, w, target, dloss)
    there = (target >= 0).cuda()
    assert not bool(loss[~there].any()) and not bool(r["dh"][~there].any())


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_what_is_not_finite_stays_in_its_row(api, io):
    import torch
    h, w, target, dloss = _make(2, 40, 300, 64, io)
    clean = _both(api, h, w, target, dloss)
    target[7], target[9] = -1, -5
    without = _both(api, h, w, target, dloss)
    h[7], h[9], dloss[9] = float("nan"), float("inf"), float("nan")              # rows without a target
    loss, lse = api.lrnnx_vocab_loss_fwd(h.cuda(), w.cuda(), target.cuda())
    r = api.lrnnx_vocab_loss_bwd(h.cuda(), w.cuda(), target.cuda(), lse, dloss.cuda())
    keep = [i for i in range(40) if i not in (7, 9)]
    assert torch.equal(loss, without[0]) and torch.equal(lse[keep], without[1][keep])
    assert torch.equal(r["dh"], without[2]["dh"]) and torch.equal(r["dweight"], without[2]["dweight"])
    h, w, target, dloss = _make(2, 40, 300, 64, io)
    target[3] = 300                                        # beyond the vocabulary: its row is lost, no other
    loss, lse = api.lrnnx_vocab_loss_fwd(h.cuda(), w.cuda(), target.cuda())
    r = api.lrnnx_vocab_loss_bwd(h.cuda(), w.cuda(), target.cuda(), lse, dloss.cuda())
    keep = [i for i in range(40) if i != 3]
    assert torch.equal(loss[keep], clean[0][keep]) and torch.equal(lse, clean[1]) and bool(torch.isnan(loss[3]))
    assert torch.equal(r["dh"][keep], clean[2]["dh"][keep]) and bool(torch.isnan(r["dh"][3]).all()) and bool(torch.isnan(r["dweight"]).all())


def test_logits_far_apart(api):
    import torch
    w = torch.zeros(600, 8, dtype=torch.bfloat16)
    w[:, 0] = torch.linspace(-300, 300, 600)
    h = torch.zeros(3, 8, dtype=torch.bfloat16)
    h[0, 0], h[1, 0], h[2, 0] = 1.0, -256.0, 0.0
    target = torch.tensor([599, 5, 17])
    _both(api, h, w, target, torch.ones(3))


def test_strided_rows_and_one_gradient(api):
    import torch
    for io in ("f32", "bf16"):
        h, w, target, dloss = (t.cuda() for t in _make(3, 24, 520, 72, io))
        loss, lse = api.lrnnx_vocab_loss_fwd(h, w, target)
        want = api.lrnnx_vocab_loss_bwd(h, w, target, lse, dloss)
        for room, at in ((80, 8), (100, 3)):
            hs, ws = (torch.full((t.shape[0], room), float("nan"), dtype=t.dtype, device="cuda")[:, at:at + 72] for t in (h, w))
            hs.copy_(h)
            ws.copy_(w)
            l2, e2 = api.lrnnx_vocab_loss_fwd(hs, ws, target)
            assert torch.equal(l2, loss) and torch.equal(e2, lse)
            one = api.lrnnx_vocab_loss_bwd(hs, ws, target, lse, dloss, want_dweight=False)
            other = api.lrnnx_vocab_loss_bwd(hs, ws, target, lse, dloss, want_dh=False)
            assert set(one) == {"dh"} and set(other) == {"dweight"}
            assert torch.equal(one["dh"], want["dh"]) and torch.equal(other["dweight"], want["dweight"])
        l3, e3 = api.lrnnx_vocab_loss_fwd(h.view(4, 6, 72), w, target.view(4, 6))
        assert l3.shape == (4, 6) and torch.equal(l3.view(24), loss)
        mean = torch.full((), 0.125, device="cuda").expand(24)
        full = api.lrnnx_vocab_loss_bwd(h, w, target, lse, mean.contiguous())
        assert all(torch.equal(v, full[n]) for n, v in api.lrnnx_vocab_loss_bwd(h, w, target, lse, mean).items())


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_reproducible_on_another_stream_and_in_a_graph(api, io):
    import torch
    h, w, target, dloss = (t.cuda() for t in _make(5, 300, 700, 100, io))

    def run():
        loss, lse = api.lrnnx_vocab_loss_fwd(h, w, target)
        return [loss, lse, *api.lrnnx_vocab_loss_bwd(h, w, target, lse, dloss).values()]
    first = run()
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
        h.copy_(torch.randn(h.shape, device="cuda"))
        target.copy_(torch.randint(-200, 700, target.shape, device="cuda"))       # another number of rows with a target
        want = run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want)), i


def test_gradients_are_differences(api):
    """Central differences of the loss in float32 along random directions: the loss is off by 2e-6 of 30 rows' sum (about 1e-4 at a step of 0.05 either way: 1e-3 of the
    difference quotient, whose curvature adds as much)."""
    import torch
    h, w, target, dloss = _make(6, 30, 400, 48, "f32")
    run = lambda a, b: (api.lrnnx_vocab_loss_fwd(a.cuda(), b.cuda(), target.cuda())[0].double().cpu() * dloss).sum()
    lse = api.lrnnx_vocab_loss_fwd(h.cuda(), w.cuda(), target.cuda())[1]
    r = api.lrnnx_vocab_loss_bwd(h.cuda(), w.cuda(), target.cuda(), lse, dloss.cuda())
    for n, t in (("dh", h), ("dweight", w)):
        d = r[n].cpu() / r[n].cpu().norm()                 # along the gradient itself
        step = 0.05
        up, down = ((h + s * d, w) if n == "dh" else (h, w + s * d) for s in (step, -step))
        want = (r[n].cpu().double() * d).sum()
        assert abs((run(*up) - run(*down)) / (2 * step) - want) < 4e-3 * want, n


@pytest.mark.parametrize("io,K", [("bf16", 64), ("bf16", 61), ("f32", 40)])
def test_a_vocabulary_in_pieces(api, io, K):
    """Rows and words whose dz does not lie in the workspace at once: the reference is taken on the GPU, in 64 bits."""
    import torch
    T, V = (16384, 33300) if io == "bf16" else (8192, 22100)
    h, w, target, dloss = (t.cuda() for t in _make(8, T, V, K, io))
    loss, lse = api.lrnnx_vocab_loss_fwd(h, w, target)
    r = api.lrnnx_vocab_loss_bwd(h, w, target, lse, dloss)
    hd, wd = h.double(), w.double()
    want = dict(loss=torch.zeros(T, dtype=torch.float64, device="cuda"), lse=torch.zeros(T, dtype=torch.float64, device="cuda"), dh=torch.zeros_like(hd), dweight=torch.zeros_like(wd))
    for lo in range(0, T, 2048):
        rows, t = slice(lo, lo + 2048), target[lo:lo + 2048]
        z = hd[rows] @ wd.t().contiguous()
        want["lse"][rows] = torch.logsumexp(z, 1)
        there = t >= 0
        pick = z.gather(1, t.clamp(min=0)[:, None])[:, 0]
        want["loss"][rows] = torch.where(there, want["lse"][rows] - pick, 0.0)
        dz = torch.exp(z - want["lse"][rows, None])
        dz.scatter_add_(1, t.clamp(min=0)[:, None], torch.full((len(t), 1), -1.0, dtype=torch.float64, device="cuda"))
        dz *= torch.where(there, dloss[rows].double(), 0.0)[:, None]
        want["dh"][rows] = dz @ wd
        want["dweight"] += dz.t().contiguous() @ hd[rows]
    for n, got in dict(r, loss=loss, lse=lse).items():
        _check(got, want[n].cpu(), n)


def test_a_copied_vocabulary_in_pieces(api):
    """Rows that cannot be read in place, and whose copy is larger than the workspace may be: forward and backward, 64 bits on the GPU."""
    import torch
    T, V, K = 3, 108000, 5001
    g = torch.Generator(device="cuda").manual_seed(1)
    w = (torch.randn(V, K, generator=g, device="cuda") * K ** -0.5).bfloat16()
    h = torch.randn(T, K, generator=g, device="cuda").bfloat16()
    target, dloss = torch.tensor([107999, -1, 5], device="cuda"), torch.tensor([1.0, 2.0, 0.5], device="cuda")
    loss, lse = api.lrnnx_vocab_loss_fwd(h, w, target)
    r = api.lrnnx_vocab_loss_bwd(h, w, target, lse, dloss)
    z = h.double() @ w.double().t().contiguous()
    want = torch.logsumexp(z, 1)
    dz = torch.exp(z - want[:, None])
    dz[0, 107999] -= 1
    dz[2, 5] -= 1
    dz *= torch.tensor([1.0, 0.0, 0.5], device="cuda", dtype=torch.float64)[:, None]
    _check(lse, want.cpu(), "lse", 5e-6)          # sums of 5001 products: 6e-8 * sqrt(5001 / 32) * 4 of a logit
    _check(r["dh"], (dz @ w.double()).cpu(), "dh")
    _check(r["dweight"], (dz.t().contiguous() @ h.double()).cpu(), "dweight")


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,K", [(90, 67, 1333), (1, 60, 4100), (3, 2500, 2050), (300, 40, 1030), (60, 1025, 600), (1100, 9, 520), (512, 260, 132), (513, 260, 132),
                                   (520, 300, 70), (130, 2100, 772)])
def test_long_sums_of_few_tiles(api, io, T, V, K):
    """Logits of up to 4100 terms, in stretches of them: 6e-8 * sqrt(4100 / 32) = 7e-7 of the largest logit, up to 7, in one chain: beside lse, which is as large, under 2e-6, and
    a factor of up to 1 + 5e-6 of an exponential."""
    _both(api, *_make(T + V + K, T, V, K, io))


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_long_sums_masks_and_strides(api, io):
    """What is not finite, targets beyond the vocabulary and views, where the logits are summed in stretches."""
    import torch
    h, w, target, dloss = _make(4, 24, 300, 520, io)
    clean = _both(api, h, w, target, dloss)
    bad = h.clone()
    bad[5], bad[6] = float("inf"), float("nan")
    target[5] = target[6] = -1
    target[8] = 300
    for at, room in ((8, 540), (3, 541)):
        hs, ws = (torch.full((t.shape[0], room), float("nan"), dtype=t.dtype, device="cuda")[:, at:at + 520] for t in (bad, w))
        hs.copy_(bad)
        ws.copy_(w)
        loss, lse = api.lrnnx_vocab_loss_fwd(hs, ws, target.cuda())
        others = [t for t in range(24) if t not in (5, 6, 8)]
        assert torch.equal(loss[others], clean[0][others]) and torch.equal(lse[others], clean[1][others])
        assert not bool(loss[5:7].any()) and bool(loss[8].isnan())
        r = api.lrnnx_vocab_loss_bwd(hs, ws, target.cuda(), lse, dloss.cuda())
        assert not bool(r["dh"][5:7].any()) and bool(r["dh"][8].isnan().all()) and bool(r["dweight"].isnan().all())
        assert torch.equal(r["dh"][others], clean[2]["dh"][others])
    target[8] = 299
    want = vocab(h[[t for t in range(24) if t not in (5, 6)]].double(), w.double(), target[[t for t in range(24) if t not in (5, 6)]],
                 dloss[[t for t in range(24) if t not in (5, 6)]].double())
    loss, lse = api.lrnnx_vocab_loss_fwd(bad.cuda(), w.cuda(), target.cuda())
    _check(api.lrnnx_vocab_loss_bwd(bad.cuda(), w.cuda(), target.cuda(), lse, dloss.cuda())["dweight"], want[3], "dweight")


def test_long_sums_of_a_vocabulary_in_pieces(api):
    """Rows of over a million terms that cannot be read in place, two pieces of words: the reference on the GPU, in 64 bits.  A logit in one chain of additions of 32 terms: 6e-8 *
    sqrt(2^20 / 32) = 1.1e-5 of it (up to 7)."""
    import torch
    T, V, K = 3, 300, (1 << 20) - 1
    g = torch.Generator(device="cuda").manual_seed(1)
    w = torch.randn(V, K, generator=g, device="cuda") * K ** -0.5
    h = torch.randn(T, K, generator=g, device="cuda") * 2
    target, dloss = torch.tensor([299, -1, 5], device="cuda"), torch.tensor([1.0, 2.0, 0.5], device="cuda")
    loss, lse = api.lrnnx_vocab_loss_fwd(h, w, target)
    r = api.lrnnx_vocab_loss_bwd(h, w, target, lse, dloss)
    hd, wd = h.double(), w.double()
    z = hd @ wd.t().contiguous()
    want = torch.logsumexp(z, 1)
    _check(lse, want.cpu(), "lse", 1.1e-5)
    _check(loss, torch.stack([want[0] - z[0, 299], want[1] * 0, want[2] - z[2, 5]]).cpu(), "loss", 3e-5)
    dz = torch.exp(z - want[:, None])
    dz[0, 299] -= 1
    dz[2, 5] -= 1
    dz *= torch.tensor([1.0, 0.0, 0.5], device="cuda", dtype=torch.float64)[:, None]
    _check(r["dh"], (dz @ wd).cpu(), "dh", 8e-5)
    _check(r["dweight"], (dz.t().contiguous() @ hd).cpu(), "dweight", 8e-5)


@pytest.mark.parametrize("same", [False, True])
@pytest.mark.parametrize("T,V,K", [(300, 4000, 256), (2500, 54, 130), (5000, 300, 64), (70, 900, 40), (2100, 16000, 520), (4000, 2000, 1100)])
def test_gradients_in_bfloat16_are_as_exact_as_their_own_rounding(api, T, V, K, same):
    """The result's rounding: rms 2^-8 / sqrt(3) of a power of two, 1.7e-3 of normally distributed numbers.  Beside the target's element, which is 1 - p of the row's dz and kept
    whole, no p is over 0.1 here (logits within +-3) and the elements' roundings are independent: 1.7e-3 * sqrt(sum p^2) / (1 - p), under 0.35 of it even for 54 words: 1.8e-3, held to 2e-3.
    (With the target's rounded: 2.4e-3.)"""
    import torch
    g = torch.Generator(device="cuda").manual_seed(T + V)
    h = torch.randn(T, K, generator=g, device="cuda").bfloat16()
    w = (torch.randn(V, K, generator=g, device="cuda") * 0.6 * K ** -0.5).bfloat16()
    target = torch.full((T,), V // 2, device="cuda") if same else torch.randint(0, V, (T,), generator=g, device="cuda")
    target[torch.rand(T, generator=g, device="cuda") < 0.1] = -1
    dloss = torch.rand(T, generator=g, device="cuda") + 0.1
    loss, lse = api.lrnnx_vocab_loss_fwd(h, w, target)
    r = api.lrnnx_vocab_loss_bwd(h, w, target, lse, dloss)
    hd, wd, there = h.double(), w.double(), target >= 0
    dz = torch.softmax(hd @ wd.t().contiguous(), 1)
    dz[torch.arange(T, device="cuda"), target.clamp(min=0)] -= 1
    dz *= torch.where(there, dloss.double(), 0.0)[:, None]
    _check(r["dh"], (dz @ wd).cpu(), "dh", 2e-3)
    _check(r["dweight"], (dz.t().contiguous() @ hd).cpu(), "dweight", 2e-3)


def test_more_rows_than_workgroups(api):
    """2^26 rows: a wavefront a row would be 2^32 threads.  Logits of 8 products of numbers up to 5: under 5e-6; lse of 5 of them."""
    import torch
    T, V, K = (1 << 26) + 3, 5, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    h = torch.randn(T, K, generator=g, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(V, K, generator=g, device="cuda").bfloat16()
    target = torch.randint(-1, V, (T,), generator=g, device="cuda")
    loss, lse = api.lrnnx_vocab_loss_fwd(h, w, target)
    for rows in (slice(0, 1000), slice(1 << 25, (1 << 25) + 1000), slice(T - 1000, T)):
        z = h[rows].double() @ w.double().t().contiguous()
        want, t = torch.logsumexp(z, 1), target[rows]
        pick = torch.where(t >= 0, want - z.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)
        assert float((lse[rows].double() - want).abs().max()) < 5e-6 and float((loss[rows].double() - pick).abs().max()) < 1e-5


@pytest.mark.parametrize("T,V,K", [(1, 300, 65), (9, 9000, 981), (70, 700, 1333), (300, 771, 203), (512, 2100, 133)])
def test_float32_rows_anywhere(api, T, V, K):
    """Few rows in float32 read the words as they lie, an element at a time where those are no 16-byte pieces: any start and step gives the same numbers, and nothing beside a row is read."""
    import torch
    h, w, target, dloss = _make(T + K, T, V, K, "f32")
    loss, lse, r = _both(api, h, w, target, dloss)
    for at, room in ((1, K + 1), (2, K + 7), (0, K + 3)):
        wide = torch.full((V, room), float("nan"), device="cuda")
        ws = wide[:, at:at + K]
        ws.copy_(w)
        l2, e2 = api.lrnnx_vocab_loss_fwd(h.cuda(), ws, target.cuda())
        r2 = api.lrnnx_vocab_loss_bwd(h.cuda(), ws, target.cuda(), e2, dloss.cuda())
        assert torch.equal(l2, loss) and torch.equal(e2, lse) and all(torch.equal(r[n], r2[n]) for n in r)


def test_words_that_are_one_row(api):
    """Rows a step of 0 apart (copied first)."""
    import torch
    for io in ("f32", "bf16"):
        h, w, target, dloss = (t.cuda() for t in _make(1, 20, 300, 72, io, none=0.0))
        w = w[:1].expand(300, 72)
        loss, lse = api.lrnnx_vocab_loss_fwd(h, w, target)
        want = vocab(h.cpu().double(), w.cpu().double(), target.cpu(), dloss.cpu().double())
        _check(loss, want[0], "loss")
        r = api.lrnnx_vocab_loss_bwd(h, w, target, lse, dloss)
        _check(r["dweight"], want[3], "dweight")
        assert float(r["dh"].abs().max()) < 1e-5           # the formula's is 0


@pytest.mark.parametrize("T,V,K", [(512, 300, 255), (513, 300, 255), (576, 700, 256), (577, 700, 260), (768, 300, 259), (769, 2100, 256), (640, 7000, 333)])
def test_float32_words_split_where_read_or_copied(api, T, V, K):
    """Either side of where either pass goes over from one to the other, and one each."""
    _both(api, *_make(T + K, T, V, K, "f32"))
