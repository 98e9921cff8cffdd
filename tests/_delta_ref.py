"""Plain references in 64 bits for the gated delta rule and the norms around a block: numpy, one step after the other, no code of the
library."""
import numpy as np


def _heads(x, share):
    return np.repeat(x, share, axis=-2)


def delta_fwd(q, k, v, g, beta, scale, s0=None):
    """o [L,Hv,dv], states [L+1,Hv,dk,dv] (states[t]: before step t), corrections e [L,Hv,dv]; one sequence, [L,H,..] float64 inputs."""
    L, Hk, dk = q.shape
    Hv, dv = v.shape[1:]
    q, k = _heads(q, Hv // Hk), _heads(k, Hv // Hk)
    S = np.zeros((Hv, dk, dv)) if s0 is None else s0.copy()
    o, e, states = np.zeros((L, Hv, dv)), np.zeros((L, Hv, dv)), [S]
    for t in range(L):
        S = S * np.exp(g[t])[:, None, None]
        e[t] = v[t] - (S * k[t][..., None]).sum(1)
        S = S + k[t][..., None] * (beta[t][:, None] * e[t])[:, None, :]
        o[t] = scale * (S * q[t][..., None]).sum(1)
        states.append(S)
    return o, states, e


def delta_bwd(q, k, v, g, beta, scale, do, s0=None, ds_last=None):
    """Gradients of sum(do * o) + sum(ds_last * last state): dict dq, dk, dv, dg, dbeta, ds0."""
    L, Hk, dk_ = q.shape
    Hv, dv_ = v.shape[1:]
    share = Hv // Hk
    _, states, e = delta_fwd(q, k, v, g, beta, scale, s0)
    q, k = _heads(q, share), _heads(k, share)
    dS = np.zeros_like(states[0]) if ds_last is None else ds_last.copy()
    r = dict(dq=np.zeros(q.shape), dk=np.zeros(k.shape), dv=np.zeros(v.shape), dg=np.zeros(g.shape), dbeta=np.zeros(g.shape))
    for t in reversed(range(L)):
        a, b = np.exp(g[t])[:, None, None], beta[t][:, None]
        dS = dS + scale * q[t][..., None] * do[t][:, None, :]
        r["dq"][t] = scale * (states[t + 1] * do[t][:, None, :]).sum(2)
        du = (dS * k[t][..., None]).sum(1)                       # gradient of beta e
        r["dbeta"][t] = (du * e[t]).sum(1)
        r["dv"][t] = b * du
        r["dk"][t] = (dS * (b * e[t])[:, None, :]).sum(2) - (a * states[t] * (b * du)[:, None, :]).sum(2)
        dS = dS - k[t][..., None] * (b * du)[:, None, :]         # gradient of exp(g) S
        r["dg"][t] = (dS * a * states[t]).sum((1, 2))
        dS = dS * a
    for n in ("dq", "dk"):
        r[n] = r[n].reshape(L, Hk, share, dk_).sum(2)
    return dict(r, ds0=dS)


def norm_fwd(x, post=None, groups=1, gate=None, act="silu", residual=None, scale=None, pre=None, eps=1e-6):
    """h, y and what the derivative needs; rows [M,D] float64."""
    M, D = x.shape
    c = dict(n=x, w=np.ones(D), a=np.ones((1, 1)), r1=None)
    if post is not None:
        xg = x.reshape(M, groups, D // groups)
        c["r1"] = 1 / np.sqrt((xg ** 2).mean(2, keepdims=True) + eps)
        c["n"] = (xg * c["r1"]).reshape(M, D)
        c["w"] = np.tile(post, D // post.size)
    if gate is not None:
        s = 1 / (1 + np.exp(-gate))
        c["a"], c["da"] = (s, s * (1 - s)) if act == "sigmoid" else (gate * s, s * (1 + gate * (1 - s)))
    c["m"] = c["n"] * c["w"]
    h = c["m"] * c["a"] * (1 if scale is None else scale) + (0 if residual is None else residual)
    y = None
    if pre is not None:
        c["r2"] = 1 / np.sqrt((h ** 2).mean(1, keepdims=True) + eps)
        c["n2"] = h * c["r2"]
        y = c["n2"] * pre
    return h, y, c


def norm_bwd(dh, dy, x, post=None, groups=1, gate=None, act="silu", residual=None, scale=None, pre=None, eps=1e-6):
    M, D = x.shape
    _, _, c = norm_fwd(x, post, groups, gate, act, residual, scale, pre, eps)
    r = {}
    dh = np.zeros_like(x) if dh is None else dh
    if pre is not None:
        dy = np.zeros_like(x) if dy is None else dy
        r["dpre_weight"] = (dy * c["n2"]).sum(0)
        dn = dy * pre
        dh = dh + c["r2"] * (dn - c["n2"] * (dn * c["n2"]).mean(1, keepdims=True))
    if residual is not None:
        r["dresidual"] = dh
    dp = dh
    if scale is not None:
        r["dres_scale"], dp = (dh * c["m"] * c["a"]).sum(0), dh * scale
    if gate is not None:
        r["dgate"] = dp * c["m"] * c["da"]
    dm = dp * c["a"]
    if post is not None:
        r["dpost_weight"] = (dm * c["n"]).sum(0).reshape(-1, post.size).sum(0)
        dn, n = (dm * c["w"]).reshape(M, groups, -1), c["n"].reshape(M, groups, -1)
        dm = (c["r1"] * (dn - n * (dn * n).mean(2, keepdims=True))).reshape(M, D)
    return dict(r, dx=np.broadcast_to(dm, x.shape))
