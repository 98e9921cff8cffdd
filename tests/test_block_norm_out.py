"""CPU checks of the binding's own refusals for a caller's output of the norms around a block: an `out` of another type than h's is refused before
anything is handed to the library (which takes h's element size from the residual's type, so a narrower buffer would be written past its end)."""
import pytest


@pytest.fixture()
def call(monkeypatch):
    """The Python function behind the device check, and what it hands to the library."""
    pytest.importorskip("torch")
    from paper_2602_08810_amd import api
    handed = []
    monkeypatch.setattr(api, "_call", lambda name, args: handed.append(name) or 0)
    monkeypatch.setattr(api, "_stream", lambda: 0)
    return api.lrnnx_block_norm_fwd.__wrapped__.__wrapped__, handed


@pytest.mark.parametrize("io,res,out", [("bfloat16", "float32", "bfloat16"), ("bfloat16", "bfloat16", "float32"), ("float32", "float32", "bfloat16"),
                                        ("float32", "float32", "float64")])
def test_out_of_another_type_than_the_residual_is_refused(call, io, res, out):
    import torch
    f, handed = call
    io, res, out = (getattr(torch, t) for t in (io, res, out))
    x, r = torch.zeros(4, 96, dtype=io), torch.zeros(4, 96, dtype=res)
    with pytest.raises(TypeError):
        f(x, residual=r, out=torch.zeros(4, 96, dtype=out))
    assert not handed


@pytest.mark.parametrize("io,res,out", [("bfloat16", "float32", "float32"), ("bfloat16", "bfloat16", "bfloat16"), ("float32", "float32", "float32"),
                                        ("bfloat16", None, "float32"), ("bfloat16", None, "bfloat16"), ("float32", None, "float32")])
def test_out_of_h_s_type_is_taken(call, io, res, out):
    import torch
    f, handed = call
    io, out = getattr(torch, io), getattr(torch, out)
    x, r = torch.zeros(4, 96, dtype=io), None if res is None else torch.zeros(4, 96, dtype=getattr(torch, res))
    o = torch.zeros(4, 96, dtype=out)
    h, y = f(x, residual=r, out=o, post_weight=torch.ones(96))
    assert h is o and y is None and handed == ["lrnnx_block_norm_fwd"]


def test_out_of_another_shape_or_order_is_refused(call):
    import torch
    f, handed = call
    x = torch.zeros(4, 96)
    for out in (torch.zeros(4, 97), torch.zeros(3, 96), torch.zeros(96, 4).t()):
        with pytest.raises(ValueError):
            f(x, out=out)
    assert not handed
