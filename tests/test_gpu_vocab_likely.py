"""GPU tests of the loss over a vocabulary in bfloat16 where a row is sure of words that are not its target, and where all words have a component in common: the gradients are as
exact as their own rounding to bfloat16.

Tolerance of the 2-norm, from the exact dz of each case: the result's own rounding (taken: the exact result rounded), and, independent of it, what rounding dz leaves.  Elements of a p over
1/8 and the target's are kept whole; another's rounding is at most 2^-8 / sqrt(3) of it in the root mean square (a number at the lower end of its power of two).  To dw it counts times its row of
h, to dh times the difference between its word and the mean of the words by their p, since these are brought to the sum that they have.  A tenth on top for the finite number of elements and float32 sums."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    import torch
    assert torch.cuda.is_available()
    from paper_2602_08810_amd import api as _api
    _api.lib()
    return _api


def _make(seed, T, V, K, shared, p, words, same=False):
    """Rows that give `words` words (of one place if `same`) p in all; a component of `shared` times a word's own norm is common to all words, and moves no logit but by rounding."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.float64)
    c = rand(K)
    c *= 0.6 / c.norm()
    own = 0.6 * K ** -0.5 * rand(V, K)
    w = (own + shared * c).bfloat16()
    own = w.double() - shared * c
    h = rand(T, K)
    h -= (h @ c)[:, None] * c / (c @ c)
    sure = torch.stack([torch.randperm(V, generator=g, device="cuda")[:words] for _ in range(1 if same else min(T, 512))])
    sure = sure[torch.arange(T, device="cuda") % len(sure)]
    lse = torch.cat([torch.logsumexp(part @ own.t().contiguous(), 1) for part in h.split(2048)])
    a = own[sure]                                          # [T,words,K]
    want = torch.log(torch.tensor(p / words / (1 - p), dtype=torch.float64, device="cuda")) + lse[:, None] - torch.bmm(a, h[:, :, None])[:, :, 0]
    gram = torch.bmm(a, a.transpose(1, 2).contiguous()) + 1e-9 * torch.eye(words, dtype=torch.float64, device="cuda")
    h += torch.bmm(a.transpose(1, 2).contiguous(), torch.linalg.solve(gram, want)[:, :, None])[:, :, 0]
    target = torch.randint(0, V, (T,), generator=g, device="cuda")
    target[torch.rand(T, generator=g, device="cuda") < 0.1] = -1
    return h.bfloat16(), w, target, torch.rand(T, generator=g, device="cuda") + 0.1


def _check(api, h, w, target, dloss):
    import torch
    loss, lse = api.lrnnx_vocab_loss_fwd(h, w, target)
    r = api.lrnnx_vocab_loss_bwd(h, w, target, lse, dloss)
    hd, wd = h.double(), w.double()
    dh, dw = torch.zeros_like(hd), torch.zeros_like(wd)
    left_h, left_w = 0.0, 0.0
    norms = (wd * wd).sum(1)
    for lo in range(0, len(h), 2048):
        rows, t = hd[lo:lo + 2048], target[lo:lo + 2048]
        at, there = t.clamp(min=0)[:, None], t >= 0
        p = torch.softmax(rows @ wd.t().contiguous(), 1)
        listed = (p > 0.125).scatter(1, at, True)
        dz = p.scatter_add(1, at, torch.full((len(t), 1), -1.0, dtype=torch.float64, device="cuda")) * torch.where(there, dloss[lo:lo + 2048].double(), 0.0)[:, None]
        dh[lo:lo + 2048] = dz @ wd
        dw += dz.t().contiguous() @ rows
        left = torch.where(listed, 0.0, dz).square()
        mine = p @ wd
        left_h += (left * (norms[None] - 2 * (mine @ wd.t().contiguous()) + (mine * mine).sum(1)[:, None])).sum().item()
        left_w += (left.sum(1) * (rows * rows).sum(1)).sum().item()
    for n, want, left in (("dh", dh, left_h), ("dweight", dw, left_w)):
        own = ((want.bfloat16().double() - want).norm() / want.norm()).item()
        tol = 1.1 * (own ** 2 + (2 ** -8) ** 2 / 3 * left / want.square().sum().item()) ** 0.5
        e = ((r[n].double() - want).norm() / want.norm()).item()
        assert tol < 2.3e-3 and e <= tol, f"{n}: relative error {e:.3e}, tolerance {tol:.3e}, own rounding {own:.3e}"
    return lse, r


@pytest.mark.parametrize("shared", [0, 3, 10])
@pytest.mark.parametrize("p,words", [(0.95, 1), (0.45, 1), (0.9, 3), (0.97, 7), (0.7, 8)])
@pytest.mark.parametrize("T,V,K", [(2100, 8000, 256), (300, 2000, 264), (90, 700, 1300)])
def test_rows_sure_of_other_words(api, T, V, K, p, words, shared):
    _check(api, *_make(T + words, T, V, K, shared, p, words))


@pytest.mark.parametrize("T,V,K", [(5000, 300, 96), (2500, 54, 130), (4200, 9000, 64)])
@pytest.mark.parametrize("p,words", [(0.95, 1), (0.9, 4)])
def test_all_rows_sure_of_the_same_words(api, T, V, K, p, words):
    """More rests in one tile than a stretch of rows holds at a time."""
    h, w, target, dloss = _make(T, T, V, K, 3, p, words, same=True)
    target[::3] = torch_first = int(target[target >= 0][0])
    assert torch_first >= 0
    _check(api, h, w, target, dloss)


def test_a_vocabulary_in_pieces(api):
    _check(api, *_make(5, 16384, 33300, 64, 3, 0.9, 3))


def test_reproducible(api):
    """Rests are found in any order, and used in one."""
    import torch
    for shape in ((2100, 8000, 256), (90, 700, 1300)):
        h, w, target, dloss = _make(7, *shape, 3, 0.97, 7)
        lse = api.lrnnx_vocab_loss_fwd(h, w, target)[1]
        first = api.lrnnx_vocab_loss_bwd(h, w, target, lse, dloss)
        for _ in range(10):
            again = api.lrnnx_vocab_loss_bwd(h, w, target, lse, dloss)
            assert all(torch.equal(first[n], again[n]) for n in first)


def test_signs_and_extremes_of_the_upstream_gradient(api):
    """Negative, zero and tiny gradients of the loss; a row beyond the vocabulary among rows that are sure."""
    import torch
    h, w, target, dloss = _make(9, 700, 2000, 128, 3, 0.95, 1)
    dloss[::2] *= -1
    dloss[::5] = 0
    _check(api, h, w, target, dloss)
    _check(api, h, w, target, dloss * 1e-20)
    target[target < 0] = 3
    lse, want = _check(api, h, w, target, dloss)
    target[13] = 2000
    r = api.lrnnx_vocab_loss_bwd(h, w, target, lse, dloss)
    keep = [i for i in range(700) if i != 13]
    assert torch.equal(r["dh"][keep], want["dh"][keep]) and bool(r["dh"][13].isnan().all()) and bool(r["dweight"].isnan().all())


def test_in_a_graph(api):
    """Replays with other rows, sure of other words and of as many as before or fewer, in the same workspace."""
    import torch
    h, w, target, dloss = _make(3, 300, 2000, 264, 3, 0.97, 7)
    run = lambda: list(api.lrnnx_vocab_loss_bwd(h, w, target, api.lrnnx_vocab_loss_fwd(h, w, target)[1], dloss).values())
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for i, (p, words) in enumerate([(0.97, 7), (0.9, 3), (0.5, 8), (0.95, 1), (0.97, 7)]):
        other = _make(3, 300, 2000, 264, 3, p, words)      # (the same words, of other rows)
        for a, b in zip((h, target, dloss), (other[0], other[2], other[3])):
            a.copy_(b.roll(i, 0))
        want = run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), i
