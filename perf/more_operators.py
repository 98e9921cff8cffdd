"""The performance workload of three operators around the recurrences of a language model: the short causal convolution before
a recurrence, the loss over a vocabulary without its logits, and the global norm and clipping of a model's gradients.

A case is a dict of plain values.  `kind` selects the operator:

    conv     short causal convolution with bias and activation over a sequence, [B,L,D] ("bld") or [B,D,L] ("bdl"): `run` is
             "forward" or "train" (outputs, then the gradients of all inputs); S > 0: a packed batch of S sequences, L steps in
             all; `state`: from carried inputs on, the last ones returned
    step     one generated token of the convolution: the carried inputs are updated in place
    loss     softmax cross entropy of T rows of K elements over V words: `run` is "forward" (loss and log of the sum) or "train"
    clip     norm of all tensors of a model's gradients, and the gradients scaled to a largest norm

`listed()` gives the named cases, `draw(rng)` one more of the same ranges, `prepare(case, seed)` the tensors on the GPU,
`run(state)` one pass, `work(case)` the bytes and operations a pass cannot do without, `exact(case, seed)` the results in 64
bits.  Where `own` is false, `run` computes the same in elementary torch operations in 32 bits.
"""
import math
import random

import torch

own = False


def listed():
    return [
        # Generation for one user: a call for each token and layer, bound by the latency of one small launch.
        dict(name="step_one", kind="step", B=1, D=4096, W=4, io="bf16", bias=True, act="silu"),
        # Generation for a full batch of a wide layer.
        dict(name="step_batch", kind="step", B=256, D=8192, W=4, io="bf16", bias=True, act="silu"),
        # Prompts before a gated delta rule: q, k and v are one view of a wider projection.
        dict(name="conv_prompts", kind="conv", run="forward", layout="bld", B=4, L=2048, S=0, D=6144, W=4, io="bf16", bias=False,
             act="silu", state=True, fused=True),
        # Training step of the convolution before a selective scan, time axis contiguous.
        dict(name="conv_train_channels", kind="conv", run="train", layout="bdl", B=8, L=2048, S=0, D=1536, W=4, io="bf16",
             bias=True, act="silu", state=False, fused=False),
        # Training step of the convolution before a gated delta rule, a large batch.
        dict(name="conv_train_rows", kind="conv", run="train", layout="bld", B=4, L=4096, S=0, D=6144, W=4, io="bf16", bias=True,
             act="silu", state=False, fused=False),
        # Packed sequences that go on from carried inputs, in float32, on sizes that divide nothing.
        dict(name="conv_ragged_f32", kind="conv", run="train", layout="bld", B=1, L=4099, S=24, D=771, W=3, io="f32", bias=True,
             act="silu", state=True, fused=False),
        # Evaluation of a few prompts: the loss alone.
        dict(name="loss_eval", kind="loss", run="forward", T=512, V=32768, K=2048, io="bf16", ignored=0.3),
        # Training step's loss: all rows have a target.
        dict(name="loss_train", kind="loss", run="train", T=8192, V=32768, K=2048, io="bf16", ignored=0.0),
        # Training on answers alone over a large vocabulary: a third of the rows are the question's and have no target.
        dict(name="loss_train_large", kind="loss", run="train", T=4096, V=131072, K=2560, io="bf16", ignored=0.33),
        # All in float32 on odd sizes, a vocabulary of a small tokenizer.
        dict(name="loss_ragged_f32", kind="loss", run="train", T=997, V=5003, K=771, io="f32", ignored=0.2),
        # A small model's gradients, float32, some of a few elements: bound by latency.
        dict(name="clip_small", kind="clip", tensors=26, total=1 << 20, io="f32", out="same", reached=True),
        # Gradients of a model in bfloat16, with its norms' in float32, clipped.
        dict(name="clip_model", kind="clip", tensors=290, total=400_000_000, io="mixed", out="same", reached=True),
    ]


# ---------------------------------------------------------------- further cases of the same ranges
def _log(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["conv", "conv", "conv", "step", "loss", "loss", "clip"])
    io = rng.choice(["bf16", "bf16", "f32"])
    if kind == "step":
        D = _log(rng, 32, 16384)
        return dict(kind=kind, B=_log(rng, 1, max(1, min(1024, (1 << 21) // D))), D=D, W=rng.choice([4, 4, 3, 2]), io=io,
                    bias=rng.random() < 0.7, act=rng.choice(["silu", "silu", "none"]))
    if kind == "conv":
        D = rng.choice([_log(rng, 16, 12288), _log(rng, 2, 96) * 64])
        most = max(1, 90_000_000 // (D if io == "bf16" else 2 * D))         # time steps in all
        L = _log(rng, 1, min(65536, most))
        S = _log(rng, 1, 48) if rng.random() < 0.3 else 0
        return dict(kind=kind, run=rng.choice(["forward", "train"]), layout=rng.choice(["bld", "bdl"]),
                    B=1 if S else _log(rng, 1, max(1, min(32, most // L))), L=L, S=S, D=D, W=rng.choice([4, 4, 3, 2]), io=io,
                    bias=rng.random() < 0.7, act=rng.choice(["silu", "silu", "none"]), state=rng.random() < 0.5,
                    fused=rng.random() < 0.3, lengths=rng.randrange(1 << 16))
    if kind == "loss":
        V, K = _log(rng, 50, 160000), rng.choice([_log(rng, 16, 5120), _log(rng, 1, 40) * 128])
        run = rng.choice(["forward", "train", "train"])
        most = (1_200_000_000_000 if run == "train" else 400_000_000_000) // (8 if io == "f32" else 1)
        return dict(kind=kind, run=run, T=_log(rng, 1, max(1, min(16384, most // (V * K)))), V=V, K=K, io=io,
                    ignored=rng.choice([0.0, 0.0, rng.uniform(0.0, 1.0)]))
    tensors = _log(rng, 1, 600)
    return dict(kind=kind, tensors=tensors, total=max(tensors, _log(rng, 1000, 300_000_000)), io=rng.choice(["bf16", "f32", "mixed"]),
                out=rng.choice(["same", "same", "f32"]), reached=rng.random() < 0.7, sizes=rng.randrange(1 << 16))


# ---------------------------------------------------------------- inputs
def _shares(rng, total, count):
    """`count` whole numbers that add up to `total`, log-normal shares."""
    share = [rng.lognormvariate(0.0, 0.8) for _ in range(count)]
    edges = [round(total * sum(share[:i]) / sum(share)) for i in range(count + 1)]
    return [b - a for a, b in zip(edges, edges[1:])]


def _lengths(case):
    return _shares(random.Random(case.get("lengths", 1)), case["L"], case["S"])


def _sizes(case):
    """Elements of the gradients' tensors: half of them are vectors, of norms and biases."""
    r, n = random.Random(case.get("sizes", 1)), case["tensors"]
    small = [min(r.choice([1, 64, 128, 771, 2048, 2560, r.randint(1, 8192)]), max(1, case["total"] // (2 * n))) for _ in range(n // 2)]
    large = _shares(r, case["total"] - sum(small), n - n // 2)
    sizes = [max(1, x) for x in small + large]
    r.shuffle(sizes)
    return sizes


class _Draw:
    """Random tensors on the GPU from one seed."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda")

    def uniform(self, lo, hi, *shape):
        return torch.rand(shape, generator=self.g, device="cuda") * (hi - lo) + lo


def _io(case):
    return torch.bfloat16 if case["io"] == "bf16" else torch.float32


def _weights(case, r):
    D, W = case["D"], case["W"]
    return r.uniform(-W ** -0.5, W ** -0.5, D, W), r.uniform(-0.5, 0.5, D) if case["bias"] else None


def _prepare_conv(case, r):
    io, B, L, D, W, rows = _io(case), case["B"], case["L"], case["D"], case["W"], case["layout"] == "bld"
    lead = () if case["S"] else (B,)
    shape = (*lead, L, D) if rows else (*lead, D, L)
    s = dict(kind="conv", train=case["run"] == "train", layout=case["layout"], act=case["act"], x0=None, dx_last=None, cu=None)
    if case["fused"]:                            # a part of the channels of a wider tensor
        wide = D + D // 2 + 8
        z = r.normal(*((*lead, L, wide) if rows else (*lead, wide, L))).to(io)
        s["x"] = z[..., 8:8 + D] if rows else z[..., 8:8 + D, :]
    else:
        s["x"] = r.normal(*shape).to(io)
    s["weight"], s["bias"] = _weights(case, r)
    seqs = case["S"] or B
    if case["S"]:
        cu = [0]
        for n in _lengths(case):
            cu.append(cu[-1] + n)
        s["cu"] = torch.tensor(cu, dtype=torch.int64, device="cuda")
    if case["state"]:
        s["x0"] = r.normal(seqs, W - 1, D).to(io)
    if s["train"]:
        s["dy"] = r.normal(*shape).to(io)
        if case["state"]:
            s["dx_last"] = r.normal(seqs, W - 1, D).to(io)
    return s


def _prepare_loss(case, r):
    """Rows that point at their target with a strength of their own, so that some words are sure and some are not."""
    io, T, V, K = _io(case), case["T"], case["V"], case["K"]
    weight = (1.5 * K ** -0.5 * r.normal(V, K)).to(io)
    target = (V ** r.uniform(0.0, 1.0, T) - 1).long().clamp(0, V - 1)           # common words have low numbers
    h = (r.normal(T, K) + r.uniform(0.0, 4.0, T, 1) * weight[target].float()).to(io)
    counted = r.uniform(0.0, 1.0, T) >= case["ignored"]
    s = dict(kind="loss", train=case["run"] == "train", h=h, weight=weight, target=torch.where(counted, target, -100))
    if s["train"]:                               # of the mean over the rows with a target
        s["dloss"] = counted.float() / counted.sum().clamp(min=1)
    return s


def _flat(tensors, dtype=None):
    """One buffer for all tensors of a type, as an optimizer keeps them, each from a multiple of 64 elements on; their views."""
    flat, views = [], [None] * len(tensors)
    for t in [dtype] if dtype else sorted({t.dtype for t in tensors}, key=str):
        mine = [i for i, x in enumerate(tensors) if dtype or x.dtype == t]
        room = [-(-tensors[i].numel() // 64) * 64 for i in mine]
        flat.append(torch.zeros(sum(room), dtype=t, device="cuda"))
        for i, part in zip(mine, flat[-1].split(room)):
            views[i] = part[:tensors[i].numel()]
    return flat, views


def _prepare_clip(case, r):
    sizes = _sizes(case)
    grads = []
    for i, n in enumerate(sizes):
        io = torch.bfloat16 if case["io"] == "bf16" or (case["io"] == "mixed" and n > 8192) else torch.float32
        grads.append((r.normal(n) * (0.2 + 0.1 * (i % 7))).to(io))
    typical = 0.5 * math.sqrt(sum(sizes))
    flat, out = _flat([torch.empty_like(g) for g in grads], torch.float32 if case["out"] == "f32" else None)
    return dict(kind="clip", grads=grads, flat=flat, out=out, max_norm=0.1 * typical if case["reached"] else 10.0 * typical + 10.0)


def prepare(case, seed):
    r = _Draw(seed)
    if case["kind"] == "step":
        io, B, D = _io(case), case["B"], case["D"]
        weight, bias = _weights(case, r)
        return dict(kind="step", x=r.normal(B, D).to(io), weight=weight, bias=bias, act=case["act"],
                    state=r.normal(B, case["W"] - 1, D).to(io))
    return {"conv": _prepare_conv, "loss": _prepare_loss, "clip": _prepare_clip}[case["kind"]](case, r)


# ---------------------------------------------------------------- plain forms, in 32 bits
def _act(pre, act):
    return pre * torch.sigmoid(pre) if act == "silu" else pre


def _plain_conv(s, x, weight, bias, x0):
    """y [B,L,D] and the last inputs of [B,L,D] float32 inputs; of a packed batch [1,L,D] with the boundaries s["cu"]."""
    B, L, D = x.shape
    W = weight.shape[1]
    if s["cu"] is None:
        xp = torch.cat([x0, x], 1)
        pre = sum(weight[:, j] * xp[:, j:j + L] for j in range(W))
        last = xp[:, L:]
    else:
        cu, at = s["cu"], torch.arange(L, device="cuda")
        seq = torch.searchsorted(cu, at, right=True) - 1
        pos = at - cu[seq]
        pre = 0
        for j in range(W):
            back = W - 1 - j                     # an input so many steps ago: of this sequence, or carried
            own_, kept = x[0, (at - back).clamp(min=0)], x0[seq, (pos + j).clamp(max=W - 2)]
            pre = pre + weight[:, j] * torch.where((pos >= back)[:, None], own_, kept)
        pre = pre[None]
        n = cu[1:] - cu[:-1]
        last = []
        for i in range(W - 1):
            back = W - 1 - i
            last.append(torch.where((n >= back)[:, None], x[0, (cu[1:] - back).clamp(min=0)],
                                    x0[torch.arange(len(n), device="cuda"), (n + i).clamp(max=W - 2)]))
        last = torch.stack(last, 1)
    if bias is not None:
        pre = pre + bias
    return _act(pre, s["act"]), last


def _plain_conv_run(s):
    io, rows, packed = s["x"].dtype, s["layout"] == "bld", s["cu"] is not None
    D, W = s["weight"].shape
    seqs = s["cu"].numel() - 1 if packed else s["x"].shape[0]
    names = ["x", "weight"] + ["bias"] * (s["bias"] is not None) + ["x0"] * (s["x0"] is not None)
    t = {n: s[n].float() for n in names}
    if s["train"]:
        t = {n: v.detach().requires_grad_() for n, v in t.items()}
    x0 = t.get("x0", torch.zeros(seqs, W - 1, D, device="cuda"))
    with torch.set_grad_enabled(s["train"]):
        x = t["x"] if rows else t["x"].transpose(-1, -2)
        y, last = _plain_conv(s, x[None] if packed else x, t["weight"], t.get("bias"), x0)
        y = y[0] if packed else y
        y = y if rows else y.transpose(-1, -2)
    res = dict(y=y.detach().to(io).contiguous())
    if s["x0"] is not None:
        res["x_last"] = last.detach().to(io)
    if s["train"]:
        outs = [(y, s["dy"].float())] + ([(last, s["dx_last"].float())] if s["x0"] is not None else [])
        grads = torch.autograd.grad([a for a, _ in outs], list(t.values()), [b for _, b in outs])
        for n, g in zip(t, grads):
            res["d" + n] = g.to(s[n].dtype)
    return res


def _plain_step(s):
    D, W = s["weight"].shape
    x = torch.cat([s["state"], s["x"][:, None]], 1)
    pre = (x.float() * s["weight"].t()).sum(1)
    if s["bias"] is not None:
        pre = pre + s["bias"]
    s["state"].copy_(x[:, 1:])
    return _act(pre, s["act"]).to(s["x"].dtype), s["state"]


def _plain_loss(s):
    h, w, target = s["h"].float(), s["weight"].float(), s["target"]
    there, at = target >= 0, target.clamp(min=0)[:, None]
    z = h @ w.t()
    top = z.amax(1, keepdim=True)
    lse = torch.log(torch.exp(z - top).sum(1)) + top[:, 0]
    loss = torch.where(there, lse - z.gather(1, at)[:, 0], 0.0)
    if not s["train"]:
        return loss, lse
    dz = torch.exp(z - lse[:, None])
    del z
    dz.scatter_add_(1, at, torch.full_like(at, -1, dtype=dz.dtype))
    dz *= torch.where(there, s["dloss"], 0.0)[:, None]
    return dict(loss=loss, lse=lse, dh=(dz @ w).to(s["h"].dtype), dweight=(dz.t() @ h).to(s["weight"].dtype))


def _plain_clip(s):
    norm = torch.stack([g.double().square().sum() for g in s["grads"]]).sum().sqrt()
    scale = (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0).float()
    for g, o in zip(s["grads"], s["out"]):
        o.copy_(g.float() * scale)
    return norm.float(), s["flat"]


# ---------------------------------------------------------------- one pass
def run(s):
    if not own:
        return {"conv": _plain_conv_run, "step": _plain_step, "loss": _plain_loss, "clip": _plain_clip}[s["kind"]](s)
    from paper_2602_08810_amd import api
    if s["kind"] == "step":
        return api.lrnnx_short_conv_step(s["x"], s["weight"], s["state"], bias=s["bias"], act=s["act"]), s["state"]
    if s["kind"] == "loss":
        loss, lse = api.lrnnx_vocab_loss_fwd(s["h"], s["weight"], s["target"])
        if not s["train"]:
            return loss, lse
        return dict(api.lrnnx_vocab_loss_bwd(s["h"], s["weight"], s["target"], lse, s["dloss"]), loss=loss, lse=lse)
    if s["kind"] == "clip":
        norm = api.lrnnx_grad_norm(s["grads"])
        api.lrnnx_grad_clip(s["grads"], norm, s["max_norm"], out=s["out"])
        return norm, s["flat"]
    opts = dict(bias=s["bias"], act=s["act"], x0=s["x0"], cu_seqlens=s["cu"], layout=s["layout"])
    kept = s["x0"] is not None
    res = api.lrnnx_short_conv_fwd(s["x"], s["weight"], return_last_state=kept, **opts)
    res = dict(zip(("y", "x_last"), res)) if kept else dict(y=res)
    if s["train"]:
        res.update(api.lrnnx_short_conv_bwd(s["x"], s["weight"], s["dy"], dx_last=s["dx_last"], want_dx0=kept, **opts))
    return res


def work(case):
    es = 2 if case["io"] == "bf16" else 4
    if case["kind"] == "step":
        B, D, W = case["B"], case["D"], case["W"]
        return dict(bytes=B * D * es * 2 * W + 4 * D * (W + 1), flops=B * D * (2 * W + 5))
    if case["kind"] == "conv":
        n, W = case["B"] * case["L"] * case["D"], case["W"]
        train = case["run"] == "train"
        state = (case["S"] or case["B"]) * (W - 1) * case["D"] * es * (2 + 2 * train) if case["state"] else 0
        return dict(bytes=n * es * (4 if train else 2) + state + 4 * case["D"] * (W + 1) * (1 + train),
                    flops=n * ((6 * W + 16) if train else (2 * W + 5)))
    if case["kind"] == "loss":
        T, V, K = case["T"], case["V"], case["K"]
        train = case["run"] == "train"
        return dict(bytes=(T + V) * K * es * (1 + train) + 16 * T + 4 * T * train, flops=2 * T * V * K * (3 if train else 1))
    bytes_ = 0
    for n in _sizes(case):
        size = 2 if case["io"] == "bf16" or (case["io"] == "mixed" and n > 8192) else 4
        bytes_ += n * (size + (4 if case["out"] == "f32" else size))
    return dict(bytes=bytes_, flops=3 * case["total"])


# ---------------------------------------------------------------- the definitions in 64 bits
def _exact_conv(case, s):
    """Sequence by sequence: sums over shifted inputs, and their derivative written out."""
    D, W, L, rows = case["D"], case["W"], case["L"], case["layout"] == "bld"
    first = (lambda t: t) if rows else (lambda t: t.transpose(-1, -2))           # time before channels
    x = first(s["x"]).double().reshape(-1, L, D)
    dy = first(s["dy"]).double().reshape(-1, L, D) if s["train"] else None
    w, b = s["weight"].double(), 0.0 if s["bias"] is None else s["bias"].double()
    spans, at = [], 0
    if case["S"]:
        for n in _lengths(case):
            spans.append((0, at, n))
            at += n
    else:
        spans = [(i, 0, L) for i in range(case["B"])]
    y, dx = torch.zeros_like(x), torch.zeros_like(x)
    last = torch.zeros(len(spans), W - 1, D, dtype=torch.float64, device="cuda")
    dx0, dw, db = torch.zeros_like(last), torch.zeros_like(w), torch.zeros(D, dtype=torch.float64, device="cuda")
    for i, (row, lo, n) in enumerate(spans):
        seen = torch.zeros(W - 1 + n, D, dtype=torch.float64, device="cuda")
        if s["x0"] is not None:
            seen[:W - 1] = s["x0"][i].double()
        seen[W - 1:] = x[row, lo:lo + n]
        last[i] = seen[n:]
        pre = torch.zeros(n, D, dtype=torch.float64, device="cuda") + b
        for back in range(W):                    # the input `back` steps ago has weight W - 1 - back
            pre += seen[W - 1 - back:W - 1 - back + n] * w[:, W - 1 - back]
        sig = 1 / (1 + torch.exp(-pre))
        y[row, lo:lo + n] = pre if case["act"] == "none" else pre * sig
        if s["train"]:
            g = dy[row, lo:lo + n]
            if case["act"] == "silu":
                g = g * (sig + pre * sig * (1 - sig))
            into = torch.zeros_like(seen)
            if s["dx_last"] is not None:
                into[n:] += s["dx_last"][i].double()
            for back in range(W):
                part = slice(W - 1 - back, W - 1 - back + n)
                into[part] += g * w[:, W - 1 - back]
                dw[:, W - 1 - back] += (g * seen[part]).sum(0)
            db += g.sum(0)
            dx0[i], dx[row, lo:lo + n] = into[:W - 1], into[W - 1:]
    back = lambda t: first(t.reshape(first(s["x"]).shape))
    res = dict(y=back(y))
    if s["x0"] is not None:
        res["x_last"] = last
    if s["train"]:
        res.update(dx=back(dx), dweight=dw)
        if s["bias"] is not None:
            res["dbias"] = db
        if s["x0"] is not None:
            res["dx0"] = dx0
    return res


def _exact_loss(case, s):
    """A few rows at a time."""
    T, V = case["T"], case["V"]
    w = s["weight"].double()
    loss, lse = (torch.zeros(T, dtype=torch.float64, device="cuda") for _ in range(2))
    dh = torch.zeros(s["h"].shape, dtype=torch.float64, device="cuda") if s["train"] else None
    dw = torch.zeros_like(w) if s["train"] else None
    step = max(1, (1 << 27) // V)
    for lo in range(0, T, step):
        h, t = s["h"][lo:lo + step].double(), s["target"][lo:lo + step]
        z = torch.mm(h, w.t().contiguous())
        m = torch.max(z, 1, keepdim=True)[0]
        e = torch.exp(z - m)
        total = e.sum(1, keepdim=True)
        lse[lo:lo + step] = (m + torch.log(total))[:, 0]
        hit = torch.nonzero(t >= 0)[:, 0]
        loss[lo + hit] = lse[lo + hit] - z[hit, t[hit]]
        if s["train"]:
            dz = e / total
            dz[hit, t[hit]] -= 1
            scale = torch.zeros(len(t), 1, dtype=torch.float64, device="cuda")
            scale[hit, 0] = s["dloss"][lo:lo + step][hit].double()
            dz = dz * scale
            dh[lo:lo + step] = torch.mm(dz, w)
            dw += torch.mm(dz.t().contiguous(), h)
    return dict(loss=loss, lse=lse, dh=dh, dweight=dw) if s["train"] else (loss, lse)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "conv":
        return _exact_conv(case, s)
    if case["kind"] == "loss":
        return _exact_loss(case, s)
    if case["kind"] == "clip":
        norm = math.sqrt(math.fsum(torch.dot(d, d).item() for d in (g.double() for g in s["grads"])))
        scale = min(1.0, s["max_norm"] / (norm + 1e-6))
        flat = [torch.zeros(f.shape, dtype=torch.float64, device="cuda") for f in s["flat"]]
        for g, o in zip(s["grads"], s["out"]):
            (i,) = [i for i, f in enumerate(s["flat"]) if f.dtype == o.dtype]
            flat[i][o.storage_offset():o.storage_offset() + g.numel()] = g.double() * scale
        return norm, flat
    seen = [s["state"][:, j].double() for j in range(case["W"] - 1)] + [s["x"].double()]
    pre = sum(t * s["weight"][:, j].double() for j, t in enumerate(seen))
    if s["bias"] is not None:
        pre = pre + s["bias"].double()
    return pre / (1 + torch.exp(-pre)) if case["act"] == "silu" else pre, torch.stack(seen[1:], 1)
