"""The gated delta rule with so many heads that a wavefront holds whole columns of a state, against a plain implementation in 64 bits; packed and batched,
shared key heads.  Tolerances as derived for few heads: 2e-5 (float32), 6e-3 (bfloat16) of each tensor's norm."""
import numpy as np
import pytest

from _delta_ref import delta_bwd, delta_fwd
from _util import rel_l2

pytestmark = pytest.mark.gpu
F32, BF16 = 2e-5, 6e-3


@pytest.fixture(scope="module")
def api():
    import torch
    assert torch.cuda.is_available()
    from paper_2602_08810_amd import api as _api
    _api.lib()
    return _api


def _inputs(seed, lead, Hk, Hv, dk, dv, io):
    import torch
    rng = np.random.default_rng(seed)
    unit = lambda x: x / np.linalg.norm(x, axis=-1, keepdims=True)
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    make = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(dt).cuda()
    return [make(x) for x in (unit(rng.normal(size=(*lead, Hk, dk))), unit(rng.normal(size=(*lead, Hk, dk))), rng.normal(size=(*lead, Hv, dv)),
                              -0.2 * rng.exponential(size=(*lead, Hv)), rng.uniform(0, 1, (*lead, Hv)), rng.normal(size=(*lead, Hv, dv)))]


def _host(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("states", [False, True])
@pytest.mark.parametrize("B,L,Hk,Hv,dk,dv", [(3, 70, 48, 48, 64, 64), (2, 33, 24, 72, 128, 33), (5, 97, 14, 14, 128, 130), (9, 40, 15, 15, 40, 48)])
def test_forward_and_backward(api, io, states, B, L, Hk, Hv, dk, dv):
    import torch
    *x, do = _inputs(L, (B, L), Hk, Hv, dk, dv, io)
    rng = np.random.default_rng(1)
    s0, dl = (torch.from_numpy(0.5 * rng.normal(size=(B, Hv, dk, dv))).float().cuda() for _ in range(2))
    if states:
        o, last, saved = api.lrnnx_gated_delta_fwd(*x, s0=s0, return_last_state=True, return_saved=True)
        r = api.lrnnx_gated_delta_bwd(*x, do, saved, s0=s0, ds_last=dl, want_ds0=True)
    else:
        o, saved = api.lrnnx_gated_delta_fwd(*x, return_saved=True)
        r = api.lrnnx_gated_delta_bwd(*x, do, saved)
    tol = F32 if io == "f32" else BF16
    for b in range(B):
        one = [_host(t[b]) for t in x]
        first = _host(s0[b]) if states else None
        want_o, all_states, _ = delta_fwd(*one, dk ** -0.5, first)
        want = delta_bwd(*one, dk ** -0.5, _host(do[b]), first, _host(dl[b]) if states else None)
        assert rel_l2(_host(o[b]), want_o) < tol, "o"
        if states:
            assert rel_l2(_host(last[b]), all_states[-1]) < F32, "last state"
            assert rel_l2(_host(r["ds0"][b]), want["ds0"]) < F32, "ds0"
        for n in ("dq", "dk", "dv", "dg", "dbeta"):
            assert rel_l2(_host(r[n][b]), want[n]) < tol, n


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_packed(api, io):
    import torch
    spans = [(2, 2), (2, 3), (3, 67), (67, 200), (200, 232)]                     # steps 0 and 1 and the last five belong to no sequence
    cu = torch.tensor([2, 2, 3, 67, 200, 232], dtype=torch.int64, device="cuda")
    *x, do = _inputs(3, (237,), 20, 40, 64, 96, io)
    o, saved = api.lrnnx_gated_delta_fwd(*x, cu_seqlens=cu, return_saved=True)
    r = api.lrnnx_gated_delta_bwd(*x, do, saved, cu_seqlens=cu)
    tol = F32 if io == "f32" else BF16
    for lo, hi in spans:
        if lo == hi:
            continue
        one = [_host(t[lo:hi]) for t in x]
        want_o, _, _ = delta_fwd(*one, 64 ** -0.5)
        want = delta_bwd(*one, 64 ** -0.5, _host(do[lo:hi]))
        assert rel_l2(_host(o[lo:hi]), want_o) < tol, "o"
        for n in ("dq", "dk", "dv", "dbeta") + (("dg",) if hi - lo > 1 else ()):
            assert rel_l2(_host(r[n][lo:hi]), want[n]) < tol, (n, lo)
        if hi - lo == 1:                                                         # no state before the only step: its decay changes nothing
            assert float(r["dg"][lo:hi].abs().max()) == 0.0
