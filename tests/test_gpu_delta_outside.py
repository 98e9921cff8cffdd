"""Gradients of a packed batch of the gated delta rule at steps outside every sequence: exact zeros, as nothing depends on them."""
import pytest

from test_gpu_gated_delta import _make, _state, api  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("Hk,Hv,dk,dv", [(2, 2, 64, 64), (1, 3, 40, 24), (2, 4, 128, 33)])
@pytest.mark.parametrize("cu,L", [([0, 50, 130], 130), ([7, 50, 130], 200), ([150, 150, 151], 700), ([130, 130], 130), ([0, 0], 70), ([600, 640], 640)])
def test_gradients_outside_are_zero(api, monkeypatch, io, Hk, Hv, dk, dv, cu, L):  # noqa: F811
    import torch
    t, do = _make(L, (L,), Hk, Hv, dk, dv, io, "io"), _make(L + 1, (L,), Hk, Hv, dk, dv, io)["v"]
    cut = torch.tensor(cu, dtype=torch.int64, device="cuda")
    _, saved = api.lrnnx_gated_delta_fwd(**t, cu_seqlens=cut, return_saved=True)
    empty = torch.empty

    def poisoned(*args, dtype=None, **kw):                       # memory that was in use before
        x = empty(*args, dtype=dtype, **kw)
        return x.fill_(float("nan")) if dtype.is_floating_point else x

    with monkeypatch.context() as m:
        m.setattr(torch, "empty", poisoned)
        r = api.lrnnx_gated_delta_bwd(**t, do=do, saved=saved, cu_seqlens=cut)
    inside = torch.zeros(L, dtype=torch.bool, device="cuda")
    inside[cu[0]:cu[-1]] = True
    for n in ("dq", "dk", "dv", "dg", "dbeta"):
        assert not bool(r[n][~inside].any()), n
        assert bool(torch.isfinite(r[n]).all()), n
    for s, (lo, hi) in enumerate(zip(cu[:-1], cu[1:])):          # and inside as if there were nothing else
        if hi > lo:
            one = {n: x[lo:hi].unsqueeze(0) for n, x in t.items()}
            _, saved = api.lrnnx_gated_delta_fwd(**one, return_saved=True)
            want = api.lrnnx_gated_delta_bwd(**one, do=do[lo:hi].unsqueeze(0), saved=saved)
            for n in want:
                a, b = r[n][lo:hi].double(), want[n][0].double()
                assert bool(((a - b).norm() <= (2e-5 if io == "f32" else 6e-3) * b.norm().clamp(min=1e-30)).all()), (n, s)
