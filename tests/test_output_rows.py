"""CPU checks of the binding's rule for a caller's strided output of the gated delta rule: rows may lie anywhere as long as none overlap."""
import pytest


@pytest.fixture(scope="module")
def api():
    pytest.importorskip("torch")
    from paper_2602_08810_amd import api as _api
    return _api


def _views():
    import torch
    B, L, H, d = 2, 5, 3, 8
    big = torch.zeros(4 * B * L * H * d)
    yield "contiguous", big[:B * L * H * d].view(B, L, H, d)
    yield "heads first", big[:B * L * H * d].view(B, H, L, d).transpose(1, 2)
    yield "a slice of a wider row", big[:B * L * (H * d + 9)].view(B, L, H * d + 9)[..., 4:4 + H * d].unflatten(-1, (H, d))
    yield "every other step, the last one the buffer's", big[:B * (2 * L - 1) * H * d].view(B, 2 * L - 1, H, d)[:, ::2]
    yield "every other head", big[:B * L * (2 * H - 1) * d].view(B, L, 2 * H - 1, d)[:, :, ::2]
    yield "rows of different entries side by side", big[:L * H * B * d].view(L, H, B, d).permute(2, 0, 1, 3)
    yield "one step", big.as_strided((B, 1, H, d), (H * d, 1, d, 1))


def test_rows_that_do_not_overlap_are_taken(api):
    for name, t in _views():
        seen = t.clone()
        t.copy_(t + 1)
        assert float((t - seen - 1).abs().max()) == 0, name                      # (a view of distinct elements)
        assert api._out_rows(t, "out", t.shape, t.dtype)[1:] == t.stride()[:-1], name


def test_rows_that_overlap_are_refused(api):
    import torch
    big = torch.zeros(1000)
    for shape, stride in (((2, 5, 3, 8), (120, 24, 7, 1)), ((2, 5, 3, 8), (120, 23, 8, 1)), ((2, 5, 3, 8), (119, 24, 8, 1)), ((2, 5, 3, 8), (0, 24, 8, 1)),
                          ((2, 5, 3, 8), (120, 0, 8, 1)), ((2, 1, 3, 8), (16, 1, 8, 1))):
        with pytest.raises(ValueError):
            api._out_rows(big.as_strided(shape, stride), "out", torch.Size(shape), torch.float32)
