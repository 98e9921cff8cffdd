"""The performance workload of the gated delta rule and of the norms around a block: what a language model with matrix-valued
recurrent states asks of this library's entry points.

A case is a dict of plain values.  `kind` selects the operator:

    delta    gated delta rule over a sequence: `run` is "prefill" (outputs and the last state) or "train" (outputs, then the
             gradients of all inputs); S > 0: a packed batch of S sequences, L steps in all
    step     one generated token of the gated delta rule: the carried state is updated in place
    norm     norm, gate and scale after a block, sum with the residual stream, norm before the next block: `run` is "forward"
             or "train"

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
        dict(name="step_one", kind="step", B=1, Hk=8, Hv=16, dk=128, dv=128, io="bf16", gates="f32"),
        # Generation for a full batch: every state is read and written once a token.
        dict(name="step_batch", kind="step", B=128, Hk=16, Hv=32, dk=128, dv=128, io="bf16", gates="f32"),
        # A short turn of a conversation that goes on from a kept state, in float32, on sizes that divide nothing.
        dict(name="prefill_short_f32", kind="delta", run="prefill", B=2, L=77, S=0, Hk=2, Hv=6, dk=44, dv=76, io="f32",
             gates="f32", state=True, fused=False),
        # Prompts of a usual batch, q, k and v views of one projection.
        dict(name="prefill", kind="delta", run="prefill", B=4, L=2048, S=0, Hk=16, Hv=16, dk=128, dv=128, io="bf16",
             gates="f32", state=False, fused=True),
        # One long document with few heads: a long time axis and little else to spread over the chip.
        dict(name="prefill_long", kind="delta", run="prefill", B=1, L=32768, S=0, Hk=4, Hv=8, dk=128, dv=128, io="bf16",
             gates="f32", state=False, fused=False),
        # Prompts of mixed lengths packed on one time axis, two value heads to a key head.
        dict(name="prefill_packed", kind="delta", run="prefill", B=1, L=16384, S=24, Hk=8, Hv=16, dk=64, dv=128,
             io="bf16", gates="f32", state=True, fused=False),
        # Training step of one layer.
        dict(name="train", kind="delta", run="train", B=4, L=4096, S=0, Hk=16, Hv=16, dk=128, dv=128, io="bf16",
             gates="io", state=False, fused=False),
        # Training in float32 on odd sizes, shared key heads, gradients into the first state and out of the last one.
        dict(name="train_ragged_f32", kind="delta", run="train", B=3, L=531, S=0, Hk=3, Hv=6, dk=40, dv=72, io="f32",
             gates="f32", state=True, fused=False),
        # Boundary of two blocks while generating: a few rows, bound by latency.
        dict(name="norm_decode", kind="norm", run="forward", M=16, D=2560, io="bf16", post="full", groups=1, gate="",
             residual="f32", scale=True, pre=True),
        # The norm and gate of each head's output, training.
        dict(name="norm_heads_train", kind="norm", run="train", M=16384, D=2048, io="bf16", post="shared", groups=16,
             gate="silu", residual="", scale=False, pre=False),
        # Boundary of two blocks, training: norm after the one, scale, residual stream in float32, norm before the next.
        dict(name="norm_boundary_train", kind="norm", run="train", M=16384, D=2560, io="bf16", post="full", groups=1,
             gate="", residual="f32", scale=True, pre=True),
        # All of it in float32 on odd sizes.
        dict(name="norm_ragged_f32", kind="norm", run="train", M=1531, D=771, io="f32", post="full", groups=3,
             gate="sigmoid", residual="io", scale=True, pre=True),
    ]


# ---------------------------------------------------------------- further cases of the same ranges
def _log(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["delta", "delta", "delta", "step", "norm", "norm"])
    if kind == "norm":
        io = rng.choice(["bf16", "bf16", "f32"])
        groups = rng.choice([1, 1, 2, 3, 8, 16, 32])
        D = max(1, _log(rng, 64, 8192) // groups) * groups
        c = dict(kind=kind, run=rng.choice(["forward", "train", "train"]), M=_log(rng, 1, max(1, min(65536, (1 << 25) // D))),
                 D=D, io=io, post=rng.choice(["full", "shared", "full", ""]), groups=groups,
                 gate=rng.choice(["silu", "sigmoid", ""]), residual=rng.choice(["f32", "io", ""]),
                 scale=rng.random() < 0.5, pre=rng.random() < 0.7)
        if not c["post"]:
            c["groups"] = 1
        if not (c["post"] or c["gate"] or c["pre"]):
            c["pre"] = True
        return c
    io = rng.choice(["bf16", "bf16", "bf16", "f32"])
    share = rng.choice([1, 1, 2, 3, 4])
    Hk = _log(rng, 1, 16)
    c = dict(kind=kind, Hk=Hk, Hv=Hk * share, dk=rng.choice([128, 128, 64, 64, 96, rng.randint(8, 128)]),
             dv=rng.choice([128, 128, 64, 64, 256, rng.randint(8, 256)]), io=io)
    each = c["Hv"] * c["dk"] * c["dv"]
    if kind == "step":
        c["gates"] = rng.choice(["f32", "io"])
        c["B"] = _log(rng, 1, max(1, min(512, (1 << 26) // each)))
        return c
    c["run"] = rng.choice(["prefill", "train"])
    train_bf16 = c["run"] == "train" and io == "bf16"
    # training in bfloat16 starts from no state and takes its gates in bfloat16, as its gradients then are
    c["gates"] = "io" if train_bf16 or io == "f32" else rng.choice(["f32", "io"])
    c["state"] = False if train_bf16 else rng.random() < 0.5
    c["fused"] = rng.random() < 0.5
    most = (1 << 33) // (1 if c["run"] == "prefill" else 4) // (4 if io == "f32" else 1) // each    # time steps in all
    c["L"] = _log(rng, 1, max(1, min(16384, most)))
    c["S"] = _log(rng, 1, 32) if rng.random() < 0.25 else 0
    c["B"] = 1 if c["S"] else _log(rng, 1, max(1, min(16, most // c["L"])))
    c["lengths"] = rng.randrange(1 << 16)
    return c


# ---------------------------------------------------------------- inputs
def _lengths(case):
    """Lengths of the packed sequences: log-normal shares of the steps, none of them fixed to be long."""
    r = random.Random(case.get("lengths", 1))
    share = [r.lognormvariate(0.0, 0.8) for _ in range(case["S"])]
    edges = [round(case["L"] * sum(share[:i]) / sum(share)) for i in range(case["S"] + 1)]
    return [b - a for a, b in zip(edges, edges[1:])]


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


def _unit(x):
    return x / (x.square().sum(-1, keepdim=True).sqrt() + 1e-6)


def _delta_inputs(case, r, lead):
    """q, k (of length one), v, decays and write strengths: some heads forget within a few steps, some within thousands."""
    io, Hk, Hv, dk, dv = _io(case), case["Hk"], case["Hv"], case["dk"], case["dv"]
    q, k, v = _unit(r.normal(*lead, Hk, dk)), _unit(r.normal(*lead, Hk, dk)), r.normal(*lead, Hv, dv)
    if case.get("fused"):
        z = torch.cat([q.flatten(-2), k.flatten(-2), v.flatten(-2)], -1).to(io)
        q, k, v = z.split([Hk * dk, Hk * dk, Hv * dv], -1)
        q, k, v = q.unflatten(-1, (Hk, dk)), k.unflatten(-1, (Hk, dk)), v.unflatten(-1, (Hv, dv))
    else:
        q, k, v = q.to(io), k.to(io), v.to(io)
    gates = io if case["gates"] == "io" else torch.float32
    rate = torch.exp(r.uniform(math.log(2e-3), math.log(2.0), Hv))
    g = (-rate * torch.nn.functional.softplus(r.normal(*lead, Hv))).to(gates)
    beta = torch.sigmoid(r.normal(*lead, Hv)).to(gates)
    return dict(q=q, k=k, v=v, g=g, beta=beta)


def prepare(case, seed):
    r = _Draw(seed)
    io = _io(case)
    if case["kind"] == "norm":
        M, D, groups = case["M"], case["D"], case["groups"]
        width = D // groups if case["post"] == "shared" else D
        s = dict(kind="norm", train=case["run"] == "train", groups=groups, gate_act=case["gate"] or "silu",
                 x=r.normal(M, D).to(io), post_weight=1 + 0.3 * r.normal(width) if case["post"] else None,
                 gate=r.normal(M, D).to(io) if case["gate"] else None, residual=None,
                 res_scale=r.uniform(0.1, 1.0, D) if case["scale"] else None,
                 pre_weight=1 + 0.3 * r.normal(D) if case["pre"] else None)
        if case["residual"]:
            s["residual"] = (2 * r.normal(M, D)).to(torch.float32 if case["residual"] == "f32" else io)
        if s["train"]:
            s["dh"] = r.normal(M, D).to(s["residual"].dtype if case["residual"] else io)
            s["dy"] = r.normal(M, D).to(io) if case["pre"] else None
        return s
    Hv, dk, dv = case["Hv"], case["dk"], case["dv"]
    if case["kind"] == "step":
        s = _delta_inputs(case, r, (case["B"],))
        return dict(s, kind="step", state=0.3 * r.normal(case["B"], Hv, dk, dv))
    seqs = case["S"] or case["B"]
    s = _delta_inputs(case, r, (case["L"],) if case["S"] else (case["B"], case["L"]))
    s.update(kind="delta", train=case["run"] == "train", s0=None, ds_last=None, cu=None)
    if case["state"]:
        s["s0"] = 0.3 * r.normal(seqs, Hv, dk, dv)
    if case["S"]:
        cu = [0]
        for n in _lengths(case):
            cu.append(cu[-1] + n)
        s["cu"], s["longest"] = torch.tensor(cu, dtype=torch.int64, device="cuda"), max(_lengths(case))
    if s["train"]:
        s["do"] = r.normal(*s["v"].shape).to(io)
        if case["state"]:
            s["ds_last"] = r.normal(seqs, Hv, dk, dv)
    return s


# ---------------------------------------------------------------- plain forms, in 32 bits
_CHUNK = 64


def _inverse(N):
    """(I + N)^-1 of strictly lower triangular N, row by row."""
    n = N.shape[-1]
    rows = torch.eye(n, device=N.device).expand(N.shape).contiguous()
    for i in range(1, n):
        rows[..., i:i + 1, :] -= N[..., i:i + 1, :i] @ rows[..., :i, :]
    return rows


def _plain_delta(q, k, v, g, beta, s0, scale):
    """o, last state of [B,L,H,...] float32 tensors with as many key heads as value heads, a chunk of steps at a time."""
    B, L, H, dk = q.shape
    C = min(_CHUNK, L)
    pad = -L % C
    q, k, v, g, beta = (torch.nn.functional.pad(t.movedim(1, 2).reshape(B, H, L, -1), (0, 0, 0, pad)).unflatten(2, (-1, C))
                        for t in (q, k, v, g, beta))                    # [B,H,chunks,C,...]
    G = g.cumsum(-2)
    low = torch.ones(C, C, device=q.device).tril()
    decay = torch.exp((G - G.transpose(-1, -2)) * low) * low
    N = beta * decay * (k @ k.transpose(-1, -2)) * low.tril(-1)
    with torch.no_grad():
        T0 = _inverse(N)
    eye = torch.eye(C, device=q.device)
    T = T0 @ (2 * eye - (eye + N) @ T0)          # the same inverse, with its derivative
    A = scale * decay * (q @ k.transpose(-1, -2))
    reads, writes, end = torch.exp(G), torch.exp(G[..., -1:, :] - G) * k, torch.exp(G[..., -1:, :])
    S, out = s0, []
    for c in range(q.shape[2]):
        u = T[:, :, c] @ (beta[:, :, c] * (v[:, :, c] - reads[:, :, c] * (k[:, :, c] @ S)))
        out.append(scale * reads[:, :, c] * (q[:, :, c] @ S) + A[:, :, c] @ u)
        S = end[:, :, c] * S + writes[:, :, c].transpose(-1, -2) @ u
    return torch.stack(out, 2).flatten(2, 3)[:, :, :L].movedim(1, 2), S


def _plain_delta_run(s):
    io, gates = s["v"].dtype, s["g"].dtype
    Hk, Hv, dk, dv = s["q"].shape[-2], s["v"].shape[-2], s["q"].shape[-1], s["v"].shape[-1]
    inputs = [s[n].float() for n in ("q", "k", "v", "g", "beta")]
    seqs = s["cu"].numel() - 1 if s["cu"] is not None else s["v"].shape[0]
    s0 = s["s0"] if s["s0"] is not None else torch.zeros(seqs, Hv, dk, dv, device="cuda")
    if s["train"]:
        inputs = [t.detach().requires_grad_() for t in inputs]
        s0 = s0.detach().requires_grad_()
    with torch.set_grad_enabled(s["train"]):
        q, k, v, g, beta = inputs
        if s["cu"] is not None:                  # one row a sequence, filled up with steps that change nothing
            cu, total = s["cu"], v.shape[0]
            at = cu[:-1, None] + torch.arange(s["longest"], device="cuda")
            there = at < cu[1:, None]
            at = at.clamp(max=total - 1)
            q, k, v, g, beta = (t[at] * there.view(*there.shape, *[1] * (t.dim() - 1)) for t in (q, k, v, g, beta))
        q, k = q.repeat_interleave(Hv // Hk, -2), k.repeat_interleave(Hv // Hk, -2)
        o, last = _plain_delta(q, k, v, g, beta, s0, dk ** -0.5)
        if s["cu"] is not None:
            o = o[there]
    if not s["train"]:
        return o.to(io), last
    loss = [(o, s["do"].float())] + ([(last, s["ds_last"])] if s["ds_last"] is not None else [])
    grads = torch.autograd.grad([a for a, _ in loss], inputs + [s0], [b for _, b in loss])
    res = dict(o=o.detach().to(io))
    for n, d, t in zip(("dq", "dk", "dv", "dg", "dbeta"), grads, (io, io, io, gates, gates)):
        res[n] = d.to(t)
    if s["s0"] is not None:
        res["ds0"], res["s_last"] = grads[5], last.detach()
    return res


def _plain_step(s):
    share = s["v"].shape[1] // s["q"].shape[1]
    q, k = (s[n].float().repeat_interleave(share, 1) for n in ("q", "k"))
    S = s["state"] * torch.exp(s["g"].float())[..., None, None]
    u = s["beta"].float()[..., None] * (s["v"].float() - (k[..., None, :] @ S)[..., 0, :])
    S = S + k[..., None] * u[..., None, :]
    s["state"].copy_(S)
    return (q.shape[-1] ** -0.5 * (q[..., None, :] @ S)[..., 0, :]).to(s["v"].dtype), s["state"]


def _rms(x, groups, eps=1e-6):
    x = x.unflatten(-1, (groups, -1))
    return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps)).flatten(-2)


def _plain_norm(s, x, post, gate, residual, scale, pre):
    m = x
    if post is not None:
        m = _rms(m, s["groups"]) * (post if post.numel() == x.shape[1] else post.repeat(s["groups"]))
    if gate is not None:
        a = torch.sigmoid(gate)
        m = m * (a if s["gate_act"] == "sigmoid" else gate * a)
    if scale is not None:
        m = m * scale
    h = m if residual is None else residual + m
    return h, None if pre is None else _rms(h, 1) * pre


def _plain_norm_run(s):
    names = ("x", "post_weight", "gate", "residual", "res_scale", "pre_weight")
    args = [None if s[n] is None else s[n].float() for n in names]
    kept = (s["residual"] if s["residual"] is not None else s["x"]).dtype
    if not s["train"]:
        h, y = _plain_norm(s, *args)
        return h.to(kept), None if y is None else y.to(s["x"].dtype)
    args = [None if t is None else t.detach().requires_grad_() for t in args]
    with torch.enable_grad():
        h, y = _plain_norm(s, *args)
    outs = [h] if y is None else [h, y]
    grads = iter(torch.autograd.grad(outs, [t for t in args if t is not None], [s["dh"].float(), s["dy"].float()][:len(outs)]
                                     if y is not None else [s["dh"].float()]))
    res = dict(h=h.detach().to(kept), y=None if y is None else y.detach().to(s["x"].dtype))
    for n, t in zip(names, args):
        if t is not None:
            res["d" + n] = next(grads).to(s[n].dtype)
    return res


# ---------------------------------------------------------------- one pass
def run(s):
    if not own:
        return {"delta": _plain_delta_run, "step": _plain_step, "norm": _plain_norm_run}[s["kind"]](s)
    from paper_2602_08810_amd import api
    if s["kind"] == "step":
        return api.lrnnx_gated_delta_step(s["q"], s["k"], s["v"], s["g"], s["beta"], s["state"]), s["state"]
    if s["kind"] == "norm":
        opts = dict(post_weight=s["post_weight"], groups=s["groups"], gate=s["gate"], gate_act=s["gate_act"],
                    residual=s["residual"], res_scale=s["res_scale"], pre_weight=s["pre_weight"])
        h, y = api.lrnnx_block_norm_fwd(s["x"], **opts)
        if not s["train"]:
            return h, y
        return dict(api.lrnnx_block_norm_bwd(s["x"], dh=s["dh"], dy=s["dy"], **opts), h=h, y=y)
    inputs = (s["q"], s["k"], s["v"], s["g"], s["beta"])
    if not s["train"]:
        return api.lrnnx_gated_delta_fwd(*inputs, s0=s["s0"], cu_seqlens=s["cu"], return_last_state=True)
    if s["s0"] is None:
        o, saved = api.lrnnx_gated_delta_fwd(*inputs, cu_seqlens=s["cu"], return_saved=True)
        return dict(api.lrnnx_gated_delta_bwd(*inputs, do=s["do"], saved=saved, cu_seqlens=s["cu"]), o=o)
    o, last, saved = api.lrnnx_gated_delta_fwd(*inputs, s0=s["s0"], cu_seqlens=s["cu"], return_last_state=True,
                                               return_saved=True)
    return dict(api.lrnnx_gated_delta_bwd(*inputs, do=s["do"], saved=saved, s0=s["s0"], ds_last=s["ds_last"],
                                          want_ds0=True, cu_seqlens=s["cu"]), o=o, s_last=last)


def work(case):
    es = 2 if case["io"] == "bf16" else 4
    if case["kind"] == "norm":
        M, D = case["M"], case["D"]
        res = {"f32": 4, "io": es, "": 0}[case["residual"]]
        gate = es if case["gate"] else 0
        bytes_ = M * D * (es + gate + res + (res or es) + (es if case["pre"] else 0))
        flops = M * D * 16
        if case["run"] == "train":               # the inputs again, dh and dy in, dx, dgate and dresidual out
            bytes_ += M * D * (es + gate + res + (res or es) + (es if case["pre"] else 0) + es + gate + res)
            flops += M * D * 32
        return dict(bytes=bytes_ + 12 * D, flops=flops)
    Hk, Hv, dk, dv = case["Hk"], case["Hv"], case["dk"], case["dv"]
    gs = es if case["gates"] == "io" else 4
    token = 2 * Hk * dk * es + 2 * Hv * dv * es + 2 * Hv * gs            # q, k, v, o, g, beta
    update = 7 * Hv * dk * dv                                            # decay, read by k, write, read by q
    state = 4 * Hv * dk * dv
    if case["kind"] == "step":
        return dict(bytes=case["B"] * (token + 2 * state), flops=case["B"] * update)
    steps, seqs = case["B"] * case["L"], case["S"] or case["B"]
    if case["run"] == "prefill":
        return dict(bytes=steps * token + seqs * state * (2 if case["state"] else 1), flops=steps * update)
    back = 4 * Hk * dk * es + 3 * Hv * dv * es + 4 * Hv * gs             # the inputs again, do in, five gradients out
    return dict(bytes=steps * (token + back) + seqs * state * (4 if case["state"] else 0), flops=3 * steps * update)


# ---------------------------------------------------------------- the definition in 64 bits, a step at a time
def _walk(q, k, v, g, beta, S, scale):
    """o [n,B,H,dv], the states before each step and after the last, the corrections; [n,B,H,...] inputs."""
    out, states, errs = [], [S], []
    for t in range(q.shape[0]):
        S = S * torch.exp(g[t])[..., None, None]
        e = v[t] - (S * k[t][..., None]).sum(-2)
        S = S + k[t][..., None] * (beta[t][..., None] * e)[..., None, :]
        out.append(scale * (S * q[t][..., None]).sum(-2))
        states.append(S)
        errs.append(e)
    return out, states, errs


def _exact_delta(case, s):
    Hk, Hv, dk, dv = case["Hk"], case["Hv"], case["dk"], case["dv"]
    if case["L"] * case["B"] * Hv * dk * dv * (6 if s["train"] else 1) > 4e11:
        return None
    scale, share = dk ** -0.5, Hv // Hk
    full = {n: s[n].double() for n in ("q", "k", "v", "g", "beta")}
    do = s["do"].double() if s["train"] else None
    lens = _lengths(case) if case["S"] else [case["L"]]
    o = torch.zeros(s["v"].shape, dtype=torch.float64, device="cuda")
    seqs = case["S"] or case["B"]
    last = torch.zeros(seqs, Hv, dk, dv, dtype=torch.float64, device="cuda")
    grads = {n: torch.zeros(t.shape, dtype=torch.float64, device="cuda") for n, t in full.items()} if s["train"] else None
    ds0 = torch.zeros_like(last)
    start = 0
    for i, n in enumerate(lens):                 # sequences of a packed batch one after the other, a batch together
        rows = slice(i, i + 1) if case["S"] else slice(0, seqs)
        cut = (lambda t: t[None, start:start + n].movedim(1, 0)) if case["S"] else (lambda t: t.movedim(1, 0))
        q, k, v, g, beta = (cut(full[x]) for x in ("q", "k", "v", "g", "beta"))
        q, k = q.repeat_interleave(share, 2), k.repeat_interleave(share, 2)
        S = s["s0"][rows].double() if s["s0"] is not None else torch.zeros_like(last[rows])
        kept = []
        for c in range(0, n, 64):
            kept.append(S)
            got, states, _ = _walk(q[c:c + 64], k[c:c + 64], v[c:c + 64], g[c:c + 64], beta[c:c + 64], S, scale)
            S = states[-1]
            cut(o)[c:c + 64] = torch.stack(got)
        last[rows] = S
        if s["train"]:
            dS = s["ds_last"][rows].double() if s["ds_last"] is not None else torch.zeros_like(S)
            d = cut(do)
            into = {x: cut(grads[x]) for x in grads}
            for c in reversed(range(0, n, 64)):
                part = [t[c:c + 64] for t in (q, k, v, g, beta)]
                _, states, errs = _walk(*part, kept[c // 64], scale)
                for t in reversed(range(part[0].shape[0])):
                    qt, kt, bt, a = part[0][t], part[1][t], part[4][t], torch.exp(part[3][t])
                    dS = dS + scale * qt[..., None] * d[c + t][..., None, :]
                    dq = scale * (states[t + 1] * d[c + t][..., None, :]).sum(-1)
                    du = (dS * kt[..., None]).sum(-2)
                    de = bt[..., None] * du
                    dk_ = (dS * (bt[..., None] * errs[t])[..., None, :]).sum(-1)
                    dS = dS - kt[..., None] * de[..., None, :]
                    dk_ = dk_ - a[..., None] * (states[t] * de[..., None, :]).sum(-1)
                    into["g"][c + t] = a * (dS * states[t]).sum((-2, -1))
                    into["beta"][c + t], into["v"][c + t] = (du * errs[t]).sum(-1), de
                    into["q"][c + t] = dq.unflatten(1, (Hk, share)).sum(2)
                    into["k"][c + t] = dk_.unflatten(1, (Hk, share)).sum(2)
                    dS = dS * a[..., None, None]
            ds0[rows] = dS
        start += n
    if not s["train"]:
        return o, last
    res = dict(o=o, **{"d" + n: t for n, t in grads.items()})
    return dict(res, ds0=ds0, s_last=last) if s["s0"] is not None else res


def _exact_norm(case, s):
    """The norms and their derivatives written out."""
    M, D, G = case["M"], case["D"], case["groups"]
    d = {n: None if s.get(n) is None else s[n].double() for n in
         ("x", "post_weight", "gate", "residual", "res_scale", "pre_weight", "dh", "dy")}
    wide = None if d["post_weight"] is None else d["post_weight"].repeat(D // d["post_weight"].numel())
    if wide is not None:
        xg = d["x"].reshape(M, G, D // G)
        r1 = 1 / torch.sqrt((xg ** 2).mean(2) + 1e-6)
        n1 = (xg * r1[:, :, None]).reshape(M, D)
        m = n1 * wide
    else:
        m = d["x"]
    act = dact = None
    if d["gate"] is not None:
        sig = 1 / (1 + torch.exp(-d["gate"]))
        act, dact = (sig, sig * (1 - sig)) if case["gate"] == "sigmoid" else (d["gate"] * sig, sig * (1 + d["gate"] * (1 - sig)))
    p = m if act is None else m * act
    t = p if d["res_scale"] is None else p * d["res_scale"]
    h = t if d["residual"] is None else d["residual"] + t
    y = None
    if d["pre_weight"] is not None:
        r2 = 1 / torch.sqrt((h ** 2).mean(1, keepdim=True) + 1e-6)
        n2 = h * r2
        y = n2 * d["pre_weight"]
    if not s["train"]:
        return h, y
    dh, res = d["dh"], dict(h=h, y=y)
    if y is not None:
        res["dpre_weight"] = (d["dy"] * n2).sum(0)
        dn = d["dy"] * d["pre_weight"]
        dh = dh + r2 * (dn - n2 * (dn * n2).mean(1, keepdim=True))
    if d["residual"] is not None:
        res["dresidual"] = dh
    dp = dh
    if d["res_scale"] is not None:
        res["dres_scale"], dp = (dh * p).sum(0), dh * d["res_scale"]
    dm = dp
    if act is not None:
        res["dgate"], dm = dp * m * dact, dp * act
    if wide is not None:
        res["dpost_weight"] = (dm * n1).sum(0).reshape(-1, d["post_weight"].numel()).sum(0)
        dn = (dm * wide).reshape(M, G, D // G)
        ng = n1.reshape(M, G, D // G)
        dm = (r1[:, :, None] * (dn - ng * (dn * ng).mean(2, keepdim=True))).reshape(M, D)
    res["dx"] = dm
    return res


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        return _exact_norm(case, s)
    if case["kind"] == "delta":
        return _exact_delta(case, s)
    share = case["Hv"] // case["Hk"]
    q, k = (s[n].double().repeat_interleave(share, 1) for n in ("q", "k"))
    out, states, _ = _walk(q[None], k[None], s["v"].double()[None], s["g"].double()[None], s["beta"].double()[None],
                           s["state"].double(), case["dk"] ** -0.5)
    return out[0], states[1]
