"""GPU tests of the short causal convolution at sizes that run its main loops (many tiles, visits and slots to a thread), against the formulas in 64 bits on the GPU, sequence by
sequence, with the gradients of automatic differentiation.

Tolerances, of the 2-norm of each tensor.  y and dx: nine or ten roundings of 2^-24, as at small sizes 1e-6; rounded to bfloat16 at most 2^-8 of each element, 4e-3.  The weights'
gradients: terms off by 1e-6, added in chains of at most 1000 (steps that a thread takes, then lanes, workgroups' parts), whose roundings are independent: 6e-8 * sqrt(1000) = 2e-6, together 3e-6 of the
sum's size where terms do not cancel; dy and x are independent, so that a sum of n terms is about sqrt(n) of one, and so is what the chains' roundings add up to."""
import pytest

from _conv_regimes import CASES, boundaries
from test_gpu_short_conv import api  # noqa: F401

pytestmark = pytest.mark.gpu


def _reference(x, w, b, x0, cu):
    """y, x_last of [B,L,D] in float64; outside every sequence y is 0."""
    import torch
    W = w.shape[1]

    def one(part, before):
        seen = torch.cat([before, part])
        pre = b + sum(w[:, j] * seen[j:j + len(part)] for j in range(W))
        return pre * torch.sigmoid(pre), seen[len(part):]
    if cu is None:
        parts = [one(x[i], x0[i]) for i in range(len(x))]
        return torch.stack([p[0] for p in parts]), torch.stack([p[1] for p in parts])
    parts = [one(x[0, lo:hi], x0[i]) for i, (lo, hi) in enumerate(zip(cu, cu[1:]))]
    y = torch.cat([torch.zeros_like(x[0, :cu[0]]), *(p[0] for p in parts), torch.zeros_like(x[0, cu[-1]:])])
    return y[None], torch.stack([p[1] for p in parts])


@pytest.mark.parametrize("layout,B,L,D,W,io,packed,reaches", CASES)
def test_against_64_bits(api, layout, B, L, D, W, io, packed, reaches):  # noqa: F811
    import torch
    g = torch.Generator(device="cuda").manual_seed(L + D)
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")
    rows = 1 if packed else B
    cu = boundaries(B, L, L) if packed else None
    x, dy, x0, dl = (rand(*s).to(dt) for s in ((rows, L, D), (rows, L, D), (B, W - 1, D), (B, W - 1, D)))
    w, b = rand(D, W) * 0.5, rand(D) * 0.5
    leaves = [t.double().requires_grad_() for t in (x, w, b, x0)]
    y, last = _reference(*leaves, cu)
    want = dict(zip(("dx", "dweight", "dbias", "dx0"), torch.autograd.grad([y, last], leaves, [dy.double(), dl.double()])))
    mine = lambda t: (lambda u: u[0] if packed else u)(t if layout == "bld" else t.transpose(1, 2).contiguous())
    back = lambda t: (lambda u: u if layout == "bld" else u.transpose(1, 2))(t[None] if packed else t)
    opts = dict(bias=b, x0=x0, layout=layout)
    if packed:
        opts["cu_seqlens"] = torch.tensor(cu, dtype=torch.int64, device="cuda")
    got_y, got_last = api.lrnnx_short_conv_fwd(mine(x), w, return_last_state=True, out=torch.zeros_like(mine(x)), **opts)
    got = api.lrnnx_short_conv_bwd(mine(x), w, mine(dy), dx_last=dl, want_dx0=True, **opts)
    assert torch.equal(got_last.double(), last.detach())
    for n, t, ref in [("y", back(got_y), y.detach()), ("dx", back(got["dx"]), want["dx"]), *((n, got[n], want[n]) for n in ("dweight", "dbias", "dx0"))]:
        tol = 4e-3 if t.dtype == torch.bfloat16 else 3e-6 if n in ("dweight", "dbias") else 1e-6
        e = ((t.double() - ref).norm() / ref.norm()).item()
        assert e <= tol, f"{n}: relative error {e:.2e}, tolerance {tol:g}"
        # an error of a few elements would not show in the norm: none is off by more than roundings of its own terms
        far = ((t.double() - ref).abs() > 100 * tol * ref.abs().mean() + 2 * tol * ref.abs()).sum().item()
        assert far == 0, f"{n}: {far} elements"
