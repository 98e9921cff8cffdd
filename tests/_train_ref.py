"""Plain implementations in 64 bits of the short causal convolution, the loss over a vocabulary and the clipping of gradients, on the CPU: the
definitions, an element or a row at a time where that is what they say."""
import torch


def conv(x, w, bias, act, x0, cu=None):
    """y, x_last of x [B,L,D] (cu: [1,L,D], sequences cu[i]..cu[i+1]; y is NaN elsewhere); everything in float64, differentiable."""
    W, D = w.shape[1], w.shape[0]
    spans = [(i, 0, x.shape[1]) for i in range(x.shape[0])] if cu is None else [(0, min(max(a, 0), x.shape[1]), min(max(b, 0), x.shape[1])) for a, b in zip(cu, cu[1:])]
    y = [[None] * x.shape[1] for _ in range(x.shape[0])]
    last = []
    for i, (row, lo, hi) in enumerate(spans):
        carried = [x0[i, j] if x0 is not None else torch.zeros(D, dtype=x.dtype) for j in range(W - 1)]
        seen = carried + [x[row, t] for t in range(lo, hi)]
        for t in range(lo, hi):
            pre = torch.zeros(D, dtype=x.dtype) if bias is None else bias
            for j in range(W):
                pre = pre + w[:, j] * seen[t - lo + j]
            y[row][t] = pre * torch.sigmoid(pre) if act == "silu" else pre
        last.append(torch.stack(seen[len(seen) - (W - 1):]))
    none = torch.full((D,), float("nan"), dtype=x.dtype)
    return torch.stack([torch.stack([none if v is None else v for v in r]) for r in y]), torch.stack(last)


def vocab(h, w, target, dloss=None):
    """loss, lse and, with dloss, dh and dweight of [T,K] rows over [V,K] words."""
    z = h @ w.T
    lse = torch.logsumexp(z, 1)
    V = w.shape[0]
    loss = torch.zeros(len(h), dtype=h.dtype)
    dz = torch.zeros_like(z)
    for t, y in enumerate(target.tolist()):
        if y < 0:
            continue
        loss[t] = lse[t] - z[t, y] if y < V else float("nan")
        if dloss is not None:
            dz[t] = torch.exp(z[t] - lse[t]) if y < V else float("nan")
            if y < V:
                dz[t, y] -= 1
            dz[t] = dz[t] * dloss[t]
    if dloss is None:
        return loss, lse
    there = target >= 0                                    # rows without a target have no part in the products
    dh = torch.zeros_like(h)
    dh[there] = dz[there] @ w
    return loss, lse, dh, dz[there].T @ h[there]
