"""A small language model of gated delta rule blocks: training steps, then generation token by token from the carried states.

    y = norm(x);  q, k, v, gate, decay, strength = y W_in;  q, k, v = silu(short convolution);  o = gated delta rule;
    m = norm of each head's o, gated;  x += scale norm(m W_out);  after the last block the loss over the vocabulary

The convolution (of `conv` steps, 0: none), the recurrence, the norm and gate of the heads, the boundary between two blocks, the loss and the clipping of the
gradients are the library's calls, forward, backward and for single tokens; the dense products are torch's.  Run on an MI355X: `python examples/delta_block.py`."""
import math
import os
import sys
import time

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2602_08810_amd import api


class GatedDelta(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, g, beta):
        o, saved = api.lrnnx_gated_delta_fwd(q, k, v, g, beta, return_saved=True)
        ctx.save_for_backward(q, k, v, g, beta, saved)
        return o

    @staticmethod
    def backward(ctx, do):
        *inputs, saved = ctx.saved_tensors
        r = api.lrnnx_gated_delta_bwd(*inputs, do.contiguous(), saved)
        return r["dq"], r["dk"], r["dv"], r["dg"], r["dbeta"]


class BlockNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, post, groups, gate, residual, scale, pre):
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(x, post, gate, residual, scale, pre)
        ctx.groups = groups
        return api.lrnnx_block_norm_fwd(x, post_weight=post, groups=groups, gate=gate, residual=residual, res_scale=scale, pre_weight=pre)

    @staticmethod
    def backward(ctx, dh, dy):
        x, post, gate, residual, scale, pre = ctx.saved_tensors
        dh, dy = (None if d is None else d.contiguous() for d in (dh, dy))
        r = api.lrnnx_block_norm_bwd(x, dh, dy, post_weight=post, groups=ctx.groups, gate=gate, residual=residual, res_scale=scale, pre_weight=pre)
        return r["dx"], r.get("dpost_weight"), None, r.get("dgate"), r.get("dresidual"), r.get("dres_scale"), r.get("dpre_weight")


class ShortConv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight):
        ctx.save_for_backward(x, weight)
        return api.lrnnx_short_conv_fwd(x, weight)

    @staticmethod
    def backward(ctx, dy):
        x, weight = ctx.saved_tensors
        r = api.lrnnx_short_conv_bwd(x, weight, dy.contiguous())
        return r["dx"], r["dweight"]


class VocabLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, h, weight, target):
        loss, lse = api.lrnnx_vocab_loss_fwd(h, weight, target)
        ctx.save_for_backward(h, weight, target, lse)
        return loss

    @staticmethod
    def backward(ctx, dloss):
        h, weight, target, lse = ctx.saved_tensors
        r = api.lrnnx_vocab_loss_bwd(h, weight, target, lse, dloss.contiguous())
        return r["dh"], r["dweight"], None


def short_conv(x, weight):
    """silu of the causal convolution of x [B,L,D], a filter for every channel."""
    return ShortConv.apply(x, weight)


def vocab_loss(h, weight, target):
    """Cross entropy of every row of h [..., K] over the words of weight [V,K]; 0 where the target is negative."""
    return VocabLoss.apply(h, weight, target)


def gated_delta(q, k, v, g, beta):
    return GatedDelta.apply(q, k, v, g, beta)


def block_norm(x, post=None, groups=1, gate=None, residual=None, scale=None, pre=None):
    return BlockNorm.apply(x, post, groups, gate, residual, scale, pre)


class Model:
    """Parameters in float32 (`params`, by name), activations in `io`, the residual stream in float32."""

    def __init__(self, vocab=64, width=256, key_heads=2, value_heads=4, dk=64, dv=64, layers=2, io=torch.bfloat16, device="cuda", seed=0, conv=0):
        gen = torch.Generator().manual_seed(seed)
        self.sizes = (key_heads, value_heads, dk, dv)
        self.layers, self.io, self.conv = layers, io, conv
        self.parts = [key_heads * dk, key_heads * dk, value_heads * dv, value_heads * dv, value_heads, value_heads]
        p = dict(embed=torch.randn(vocab, width, generator=gen) * width ** -0.5, pre0=torch.ones(width))
        for i in range(layers):
            p[f"in{i}"] = torch.randn(width, sum(self.parts), generator=gen) * width ** -0.5
            p[f"out{i}"] = torch.randn(value_heads * dv, width, generator=gen) * (value_heads * dv) ** -0.5
            p[f"rate{i}"] = torch.linspace(-5.0, -1.0, value_heads)
            p[f"head{i}"], p[f"post{i}"], p[f"pre{i + 1}"] = torch.ones(dv), torch.ones(width), torch.ones(width)
            p[f"scale{i}"] = torch.full((width,), 0.5)
            if conv:
                p[f"conv{i}"] = torch.randn(sum(self.parts[:3]), conv, generator=gen) * conv ** -0.5
        self.params = {n: t.to(device).requires_grad_() for n, t in p.items()}

    def _inputs(self, i, y, convolve):
        """What the recurrence of layer i takes, from the normed residual stream: q, k, v, g, beta, and the heads' gate."""
        Hk, Hv, dk, dv = self.sizes
        z, n = y @ self.params[f"in{i}"].to(y.dtype), sum(self.parts[:3])
        q, k, v = (convolve(i, z[..., :n]) if self.conv else z[..., :n]).split(self.parts[:3], dim=-1)
        gate, a, b = z[..., n:].split(self.parts[3:], dim=-1)
        q, k = (F.normalize(t.unflatten(-1, (Hk, dk)), dim=-1) for t in (q, k))
        g = -F.softplus(a + self.params[f"rate{i}"].to(a.dtype))
        return q, k, v.unflatten(-1, (Hv, dv)), g, torch.sigmoid(b), gate

    def _run(self, tokens, recurrence, convolve):
        """The normed residual stream behind the last block."""
        p, (_, Hv, _, dv) = self.params, self.sizes
        h, y = block_norm(p["embed"][tokens].to(self.io), pre=p["pre0"])
        h = h.to(p["embed"].dtype)
        for i in range(self.layers):
            *inputs, gate = self._inputs(i, y, convolve)
            o = recurrence(i, *inputs)
            m, _ = block_norm(o.flatten(-2), post=p[f"head{i}"], groups=Hv, gate=gate)
            h, y = block_norm(m @ p[f"out{i}"].to(m.dtype), post=p[f"post{i}"], residual=h, scale=p[f"scale{i}"], pre=p[f"pre{i + 1}"])
        return y

    def _head(self, y):
        return y @ self.params["embed"].to(y.dtype).T

    def _train(self, tokens):
        return self._run(tokens, lambda i, *inputs: gated_delta(*inputs), lambda i, x: short_conv(x, self.params[f"conv{i}"]))

    def logits(self, tokens):
        """[B,L,vocab]."""
        return self._head(self._train(tokens))

    def losses(self, tokens, targets):
        """Cross entropy [B,L] of the word that follows each token, 0 where the target is negative; the logits are never in memory."""
        y = self._train(tokens)
        return vocab_loss(y, self.params["embed"].to(y.dtype), targets)

    @torch.no_grad()
    def prompt(self, tokens):
        """Logits of the prompt and the states of every layer after it."""
        states = [[None, None] for _ in range(self.layers)]

        def convolve(i, x):
            y, states[i][0] = api.lrnnx_short_conv_fwd(x, self.params[f"conv{i}"], return_last_state=True)
            return y

        def recurrence(i, *inputs):
            o, states[i][1] = api.lrnnx_gated_delta_fwd(*inputs, return_last_state=True)
            return o
        return self._head(self._run(tokens, recurrence, convolve)), states

    @torch.no_grad()
    def step(self, tokens, states):
        """Logits [B,vocab] of one more token, tokens [B]; the states move on in place."""
        return self._head(self._run(tokens, lambda i, *inputs: api.lrnnx_gated_delta_step(*inputs, states[i][1]),
                                    lambda i, x: api.lrnnx_short_conv_step(x, self.params[f"conv{i}"], states[i][0])))


def repeats(batch, length, vocab, gen):
    """Random tokens, then the same again: what a state that remembers can predict is the second half."""
    half = torch.randint(0, vocab, (batch, length), generator=gen)
    return torch.cat([half, half], 1)


def loss_of(model, tokens):
    half = tokens.shape[1] // 2
    targets = tokens[:, 1:].clone()
    targets[:, :half - 1] = -1                   # the first half cannot be known
    return model.losses(tokens[:, :-1], targets).sum() / (targets.shape[0] * (targets.shape[1] - half + 1))


def train(model, steps, batch=64, length=24, rate=5e-3, seed=1, device="cuda", every=0, clip=1.0):
    gen = torch.Generator().manual_seed(seed)
    vocab = model.params["embed"].shape[0]
    opt = torch.optim.AdamW(model.params.values(), lr=rate, weight_decay=0.0)
    losses = []
    for i in range(steps):
        loss = loss_of(model, repeats(batch, length, vocab, gen).to(device))
        opt.zero_grad()
        loss.backward()
        grads = [t.grad for t in model.params.values()]
        api.lrnnx_grad_clip(grads, api.lrnnx_grad_norm(grads), clip)
        opt.step()
        losses.append(loss.detach())
        if every and i % every == 0:
            print(f"step {i:4d}  loss {losses[-1].item():.3f}  (guessing: {math.log(vocab):.3f})", flush=True)
    return [x.item() for x in losses]


def generate(model, tokens, count):
    """Greedy continuation [B,count] of tokens [B,L]."""
    logits, states = model.prompt(tokens)
    out, logits = [], logits[:, -1]
    for _ in range(count):
        out.append(logits.argmax(-1))
        logits = model.step(out[-1], states)
    return torch.stack(out, 1)


def main():
    model = Model(vocab=32, conv=4)
    train(model, 3001, every=500)
    tokens = repeats(64, 24, model.params["embed"].shape[0], torch.Generator().manual_seed(99)).cuda()
    half = tokens.shape[1] // 2
    generate(model, tokens[:, :half + 1], 1)
    torch.cuda.synchronize()
    start = time.perf_counter()
    said = generate(model, tokens[:, :half + 1], half - 1)
    torch.cuda.synchronize()
    took = time.perf_counter() - start
    print(f"generated {said.numel()} tokens in {took * 1e3:.1f} ms, {(said == tokens[:, half + 1:]).float().mean().item():.0%} as in the first half")


if __name__ == "__main__":
    main()
