"""The example model with the short convolution, the loss over the vocabulary and the clipping: its gradients against the same model in 64 bits with plain
operators and against differences, generation against the whole sequence, and what a training step leaves.  And the convolution before the selective scan, as a
prompt and token by token.

Tolerances, of the 2-norm, as the model's without a convolution has them: 3e-4 (the convolution and the loss are right to 5e-6 and add two operators to a
dozen).  Convolution and selective scan: 1e-6 and 1e-4 of the largest number."""
import pytest

from _train_ref import conv, vocab
from test_gpu_delta_block import TOL, _plain_delta, _plain_norm, _rel, example  # noqa: F401
from _util import rel_err

pytestmark = pytest.mark.gpu


def _plain_conv(x, weight):
    return conv(x, weight, None, "silu", None)[0]


def test_gradients_are_those_of_the_plain_model(example, monkeypatch):  # noqa: F811
    import torch
    sizes = dict(vocab=23, width=96, key_heads=2, value_heads=4, dk=40, dv=24, layers=2, conv=4)
    model = example.Model(io=torch.float32, **sizes)
    tokens = example.repeats(3, 21, 23, torch.Generator().manual_seed(5))
    loss = example.loss_of(model, tokens.cuda())
    loss.backward()
    plain = example.Model(io=torch.float64, device="cpu", **sizes)
    plain.params = {n: t.detach().double().cpu().requires_grad_() for n, t in model.params.items()}
    for name, f in (("gated_delta", _plain_delta), ("block_norm", _plain_norm), ("short_conv", _plain_conv)):
        monkeypatch.setattr(example, name, f)
    half = tokens.shape[1] // 2
    logits = plain.logits(tokens[:, :-1])[:, half - 1:]
    want = torch.nn.functional.cross_entropy(logits.flatten(0, 1), tokens[:, half:].flatten())
    want.backward()
    assert abs(loss.item() - want.item()) < TOL * want.item()
    for n, t in model.params.items():
        assert _rel(t.grad, plain.params[n].grad) < TOL, n


@pytest.mark.parametrize("length", [1, 2, 3, 33])
def test_steps_go_on_where_the_prompt_ends(example, length):  # noqa: F811
    import torch
    model = example.Model(io=torch.float32, vocab=29, width=128, key_heads=1, value_heads=3, dk=64, dv=32, layers=2, conv=4)
    tokens = torch.randint(0, 29, (2, length + 6), generator=torch.Generator().manual_seed(length)).cuda()
    with torch.no_grad():
        whole = model.logits(tokens).double().cpu()
    logits, states = model.prompt(tokens[:, :length])
    assert _rel(logits, whole[:, :length]) < TOL
    for t in range(length, length + 6):
        assert _rel(model.step(tokens[:, t], states), whole[:, t]) < TOL, t


def test_a_training_step_clips_what_it_says(example):  # noqa: F811
    import torch
    model = example.Model(conv=4)
    losses = example.train(model, 3, clip=1e-3)
    assert all(x == x for x in losses)
    grads = [t.grad for t in model.params.values()]
    norm = sum(t.double().square().sum() for t in grads).sqrt().item()
    assert abs(norm - 1e-3) < 1e-3 * 0.01                   # (eps against a norm of about one, and float32)
    assert example.generate(model, example.repeats(2, 9, 64, torch.Generator().manual_seed(3)).cuda(), 5).shape == (2, 5)


def test_a_whole_step_in_a_graph(example):  # noqa: F811
    """Convolution, recurrence, loss, gradients and clipping captured together, replayed on new tokens."""
    import torch
    from paper_2602_08810_amd import api
    B, L, D, V, K = 2, 70, 96, 300, 64
    gen = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    x, w, wo, wv = rnd(B, L, D), rnd(D, 4), rnd(D, K) * 0.1, rnd(V, K) * 0.1
    target = torch.randint(-40, V, (B, L), device="cuda")
    mean = torch.full((), 1.0 / (B * L), device="cuda").expand(B, L)

    def run():
        y = api.lrnnx_short_conv_fwd(x, w)
        h = y @ wo
        loss, lse = api.lrnnx_vocab_loss_fwd(h, wv, target)
        r = api.lrnnx_vocab_loss_bwd(h, wv, target, lse, mean)
        c = api.lrnnx_short_conv_bwd(x, w, r["dh"] @ wo.t())
        grads = [c["dweight"], r["dweight"]]
        norm = api.lrnnx_grad_norm(grads)
        api.lrnnx_grad_clip(grads, norm, 0.5 * 1e-3)
        return [loss, norm, c["dx"], *grads]
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for i in range(3):
        x.copy_(rnd(B, L, D))
        target.copy_(torch.randint(-40, V, (B, L), device="cuda"))
        want = run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), i


@pytest.mark.parametrize("io", ["f32"])
def test_convolution_and_selective_scan_prompt_and_tokens(io):
    """u = silu(conv(x)) and the selective scan over it: a packed prompt of two sequences, then tokens from the carried inputs and states, against one whole sequence."""
    import torch
    from paper_2602_08810_amd import api
    D, N, lens, more = 40, 16, [37, 5], 6
    gen = torch.Generator(device="cuda").manual_seed(2)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    w, b, A, Dskip = rnd(D, 4), rnd(D), -torch.exp(rnd(D, N) * 0.3), rnd(D)
    whole = []
    for n in lens:
        n += more
        x, delta, Bm, Cm = rnd(D, n), rnd(D, n), rnd(n, N), rnd(n, N)
        u = api.lrnnx_short_conv_fwd(x[None], w, b, layout="bdl")
        y = api.lrnnx_selective_scan_fwd(u, delta[None], A, Bm[None], Cm[None], Dskip=Dskip)
        ref = conv(x.T[None].double().cpu(), w.double().cpu(), b.double().cpu(), "silu", None)[0][0].T
        assert rel_err(u[0].double().cpu(), ref) < 1e-5
        whole.append((x, delta, Bm, Cm, y[0]))
    pack = lambda i, dim: torch.cat([t[i].narrow(dim, 0, n) for t, n in zip(whole, lens)], dim).contiguous()
    cu = torch.tensor([0, lens[0], sum(lens)], dtype=torch.int64, device="cuda")
    u, inputs = api.lrnnx_short_conv_fwd(pack(0, 1), w, b, layout="bdl", cu_seqlens=cu, return_last_state=True)
    y, state = api.lrnnx_selective_scan_fwd(u, pack(1, 1), A, pack(2, 0), pack(3, 0), Dskip=Dskip, cu_seqlens=cu, return_last_state=True)
    want = pack(4, 1)
    assert rel_err(y.cpu(), want.cpu()) < 1e-4
    for t in range(more):
        at = [n + t for n in lens]
        pick = lambda i, dim: torch.stack([s[i].select(dim, a) for s, a in zip(whole, at)])
        u = api.lrnnx_short_conv_step(pick(0, 1), w, inputs, b)
        y = api.lrnnx_selective_step(state, u, pick(1, 1), A, pick(2, 0), pick(3, 0), Dskip=Dskip)
        assert rel_err(y.cpu(), pick(4, 1).cpu()) < 1e-4, t
