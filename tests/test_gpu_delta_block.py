"""The example model of gated delta rule blocks: its gradients against the same model in 64 bits with plain operators, generation against the whole
sequence, and that it learns.

Tolerances, of the 2-norm.  float32: an operator is right to 2e-5 (see the operators' own tests); about a dozen of them follow one another in two layers and
back, errors of independent sign: 2e-5 * sqrt(12) = 7e-5, and a norm's backward pass subtracts what lies along its input, so four times that: 3e-4.
Step by step against the whole sequence: both are that near to the truth: 3e-4."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
TOL = 3e-4


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "delta_block.py")
    spec = importlib.util.spec_from_file_location("delta_block", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _rel(a, b):
    return ((a.double().cpu() - b).norm() / b.norm()).item()


def _plain_delta(q, k, v, g, beta):
    import torch
    share = v.shape[2] // q.shape[2]
    q, k = (t.repeat_interleave(share, 2) for t in (q, k))
    S, out = torch.zeros(v.shape[0], v.shape[2], q.shape[3], v.shape[3], dtype=v.dtype), []
    for t in range(v.shape[1]):
        S = S * g[:, t].exp()[..., None, None]
        e = v[:, t] - (S * k[:, t][..., None]).sum(2)
        S = S + k[:, t][..., None] * (beta[:, t][..., None] * e)[:, :, None]
        out.append((S * q[:, t][..., None]).sum(2) * q.shape[3] ** -0.5)
    return torch.stack(out, 1)


def _plain_norm(x, post=None, groups=1, gate=None, residual=None, scale=None, pre=None):
    import torch
    m = x
    if post is not None:
        xg = x.unflatten(-1, (groups, -1))
        m = (xg * torch.rsqrt((xg ** 2).mean(-1, keepdim=True) + 1e-6)).flatten(-2) * post.repeat(x.shape[-1] // post.numel())
    if gate is not None:
        m = m * gate * torch.sigmoid(gate)
    h = m if scale is None else m * scale
    h = h if residual is None else h + residual
    return h, None if pre is None else h * torch.rsqrt((h ** 2).mean(-1, keepdim=True) + 1e-6) * pre


def test_gradients_are_those_of_the_plain_model(example, monkeypatch):
    import torch
    sizes = dict(vocab=23, width=96, key_heads=2, value_heads=4, dk=40, dv=24, layers=2)
    model = example.Model(io=torch.float32, **sizes)
    tokens = example.repeats(3, 41, 23, torch.Generator().manual_seed(5))
    loss = example.loss_of(model, tokens.cuda())
    loss.backward()
    plain = example.Model(io=torch.float64, device="cpu", **sizes)
    plain.params = {n: t.detach().double().cpu().requires_grad_() for n, t in model.params.items()}
    monkeypatch.setattr(example, "gated_delta", _plain_delta)
    monkeypatch.setattr(example, "block_norm", _plain_norm)
    half = tokens.shape[1] // 2
    logits = plain.logits(tokens[:, :-1])[:, half - 1:]
    want = torch.nn.functional.cross_entropy(logits.flatten(0, 1), tokens[:, half:].flatten())
    want.backward()
    assert abs(loss.item() - want.item()) < TOL * want.item()
    for n, t in model.params.items():
        assert _rel(t.grad, plain.params[n].grad) < TOL, n


@pytest.mark.parametrize("length", [1, 33, 130])
def test_steps_go_on_where_the_prompt_ends(example, length):
    import torch
    model = example.Model(io=torch.float32, vocab=29, width=128, key_heads=1, value_heads=3, dk=64, dv=32, layers=2)
    tokens = torch.randint(0, 29, (2, length + 5), generator=torch.Generator().manual_seed(length)).cuda()
    with torch.no_grad():
        whole = model.logits(tokens).double().cpu()
    logits, states = model.prompt(tokens[:, :length])
    assert _rel(logits, whole[:, :length]) < TOL
    for t in range(length, length + 5):
        assert _rel(model.step(tokens[:, t], states), whole[:, t]) < TOL, t


def test_it_learns_and_generates(example):
    import torch
    model = example.Model()
    losses = example.train(model, 60)
    assert sum(losses[-5:]) < sum(losses[:5])
    said = example.generate(model, example.repeats(4, 32, 64, torch.Generator().manual_seed(3)).cuda(), 7)
    assert said.shape == (4, 7) and int(said.min()) >= 0 and int(said.max()) < 64
