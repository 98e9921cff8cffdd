"""CPU checks: the short causal convolution refuses results that share memory with what the call reads, or with each other.  (Host code that runs before anything is
launched; the addresses are nobody's, so nothing here runs where there is a GPU that could use them.)"""
import ctypes

import pytest

from test_delta_cabi import INVALID, _call, _fill
from test_train_cabi import api  # noqa: F401

BUF, FAR = 1 << 24, 1 << 40                           # a buffer, and where everything else lies
SIZES = dict(B=2, D=96, W=4, act=0, io_dtype=1)


@pytest.fixture(autouse=True)
def no_gpu(api):  # noqa: F811
    import torch
    if torch.cuda.is_available():
        pytest.skip("addresses of no memory")


def _refused(api, name, args):  # noqa: F811
    return _call(api, name, args) == INVALID


def _seq(time_last, L=100, wide=300, x=BUF, **more):
    """x a part of a wider tensor: [2, L, wide] with 96 channels, or [2, wide, L] with rows of L steps and 3 more."""
    row = wide if not time_last else L + 3
    return {**SIZES, "time_last": time_last, "L": L, "x": x, "x_stride_b": (L if not time_last else wide) * row, "x_stride_s": row, "weight": FAR, **more}


SHIFTS = {0: [0, 2, -2, 190, -190, 300 * 2, -300 * 2, 300 * 2 + 190, 300 * 2 - 190, 99 * 600 + 40, 100 * 600, -100 * 600 + 2, 199 * 600],
          1: [0, 2, -2, 198, 206, -206, 206 + 198, 95 * 206, 300 * 206, 300 * 206 + 30 * 206 + 100, -300 * 206]}
APART = {0: [192, 196, 400, -192, -400, 408], 1: [96 * 206, -96 * 206, 200 * 206, 96 * 206 + 4, 395 * 206 + 200]}


@pytest.mark.parametrize("time_last", [0, 1])
def test_output_over_input(api, time_last):  # noqa: F811
    s = _seq(time_last)
    same = {"y_stride_b": s["x_stride_b"], "y_stride_s": s["x_stride_s"]}
    for at in SHIFTS[time_last]:
        assert _refused(api, "lrnnx_short_conv_fwd", _fill(api.ConvFwdArgs, **s, y=BUF + at, **same)), at
        for other in ("x", "dy"):
            b = {**s, "x": FAR * 2, "dy": FAR * 3, "dy_stride_b": s["x_stride_b"], "dy_stride_s": s["x_stride_s"], other: BUF, "dx": BUF + at,
                 "dx_stride_b": s["x_stride_b"], "dx_stride_s": s["x_stride_s"], "dweight": FAR * 4, "workspace": FAR * 5, "workspace_bytes": 1 << 30}
            assert _refused(api, "lrnnx_short_conv_bwd", _fill(api.ConvBwdArgs, **b)), (at, other)
    for at in APART[time_last]:                        # other channels of the same wider tensor
        assert not _refused(api, "lrnnx_short_conv_fwd", _fill(api.ConvFwdArgs, **s, y=BUF + at, **same)), at
    # steps of their own, inside the input's extent
    assert _refused(api, "lrnnx_short_conv_fwd", _fill(api.ConvFwdArgs, **s, y=BUF + 400, y_stride_b=s["x_stride_b"], y_stride_s=s["x_stride_s"] + 1))


@pytest.mark.parametrize("time_last", [0, 1])
def test_carried_inputs_and_weights(api, time_last):  # noqa: F811
    s = _seq(time_last, bias=FAR * 2, x0=FAR * 3)
    fwd = dict(s, y=FAR * 4, y_stride_b=s["x_stride_b"], y_stride_s=s["x_stride_s"])
    n, state = 2 * 300 * 103 * 2 if time_last else 2 * 100 * 300 * 2, 2 * 3 * 96 * 2
    assert not _refused(api, "lrnnx_short_conv_fwd", _fill(api.ConvFwdArgs, **fwd, x_last=FAR * 3 + state))
    for over in (dict(x_last=FAR * 3), dict(x_last=FAR * 3 + state - 2), dict(x_last=FAR * 3 - state + 2), dict(x_last=BUF + 400), dict(x_last=FAR * 4 + 1000),
                 dict(x0=FAR * 4), dict(weight=FAR * 4 + 4), dict(bias=FAR * 4 + 400), dict(x_last=FAR * 2), dict(x_last=FAR)):
        assert _refused(api, "lrnnx_short_conv_fwd", _fill(api.ConvFwdArgs, **{**fwd, **over})), over
    bwd = dict(s, dy=FAR * 4, dy_stride_b=s["x_stride_b"], dy_stride_s=s["x_stride_s"], dx_last=FAR * 5, dx=FAR * 6, dx_stride_b=s["x_stride_b"], dx_stride_s=s["x_stride_s"],
               dweight=FAR * 7, dbias=FAR * 8, dx0=FAR * 9, workspace=FAR * 10, workspace_bytes=1 << 30)
    assert not _refused(api, "lrnnx_short_conv_bwd", _fill(api.ConvBwdArgs, **bwd))
    for over in (dict(dx0=FAR * 5), dict(dx0=FAR * 3), dict(dx0=FAR * 6 + n // 4), dict(dweight=FAR), dict(dweight=FAR * 8), dict(dbias=FAR * 2), dict(dx=FAR * 3), dict(dx=FAR * 5),
                 dict(dx0=FAR * 4 + n // 8), dict(dx=FAR * 7), dict(dbias=BUF + 4)):
        assert _refused(api, "lrnnx_short_conv_bwd", _fill(api.ConvBwdArgs, **{**bwd, **over})), over


def test_packed(api):  # noqa: F811
    s = _seq(0, cu_seqlens=FAR * 2)                    # one axis of 100 steps, three sequences: batch strides mean nothing
    same = {"y_stride_b": 5, "y_stride_s": s["x_stride_s"]}
    s["B"] = 3
    assert _refused(api, "lrnnx_short_conv_fwd", _fill(api.ConvFwdArgs, **s, y=BUF + 99 * 600, **same))
    assert not _refused(api, "lrnnx_short_conv_fwd", _fill(api.ConvFwdArgs, **s, y=BUF + 100 * 600, **same))
    assert _refused(api, "lrnnx_short_conv_fwd", _fill(api.ConvFwdArgs, **{**s, "cu_seqlens": FAR * 3 + 8}, y=FAR * 3, **same))


def test_step(api):  # noqa: F811
    state = 2 * 3 * 96 * 2
    step = {**SIZES, "x": BUF, "x_stride_b": 96, "x_stride_d": 1, "weight": FAR, "bias": FAR * 2, "state": FAR * 3, "y": BUF, "y_stride_b": 96, "y_stride_d": 1}
    run = lambda **over: _refused(api, "lrnnx_short_conv_step", _fill(api.ConvStepArgs, **{**step, **over}))
    assert not run() and not run(y=FAR * 4) and not run(y=BUF + 2 * 96 * 2) and not run(state=BUF + 2 * 96 * 2)
    assert not run(x_stride_b=400, y_stride_b=400, y=BUF + 200)
    for over in (dict(y=BUF + 2), dict(y=BUF, y_stride_b=97), dict(y_stride_d=2), dict(y=FAR * 3 + state - 2), dict(x=FAR * 3, y=FAR * 4), dict(state=FAR), dict(state=FAR * 2),
                 dict(y=FAR), dict(y=FAR * 2)):
        assert run(**over), over


@pytest.mark.parametrize("time_last", [0, 1])
def test_exact_for_views_of_the_same_steps(api, time_last):  # noqa: F811
    """Against the sets of elements, on small tensors with room between rows and batch entries."""
    import random
    r = random.Random(time_last)
    met = 0
    for _ in range(600):
        B, L, D = r.randint(1, 3), r.randint(1, 4), r.randint(1, 4)
        rows, row = (D, L) if time_last else (L, D)
        ss = row + r.choice([0, 0, 1, 3, 5])
        sb = ss * (rows - 1) + row + r.choice([0, 0, 2, 7, 20])
        if r.random() < 0.3 and B > 1:                 # the batch inside
            sb, ss = row + r.choice([0, 1, 4]), 0
            ss = sb * (B - 1) + row + r.choice([0, 3, 9])
        at = r.randint(-(sb * B + ss * rows) - 2, sb * B + ss * rows + 2)
        here = {b * sb + i * ss + e for b in range(B) for i in range(rows) for e in range(row)}
        shared = any(e + at in here for e in here)
        met += shared
        a = _fill(api.ConvFwdArgs, B=B, D=D, W=2, L=L, time_last=time_last, act=0, io_dtype=1, x=BUF, x_stride_b=sb, x_stride_s=ss, weight=FAR,
                  y=BUF + 2 * at, y_stride_b=sb, y_stride_s=ss)
        assert _refused(api, "lrnnx_short_conv_fwd", a) == shared, (B, L, D, sb, ss, at)
    assert 100 < met < 500


def test_norm_among_the_results(api):  # noqa: F811
    n, kind, wide = (ctypes.c_int64 * 3)(5, 0, 100), (ctypes.c_int32 * 3)(0, 1, 1), (ctypes.c_int32 * 3)(0, 0, 0)
    grads, out = (ctypes.c_void_p * 3)(BUF, None, FAR), (ctypes.c_void_p * 3)(FAR * 2, None, FAR * 3)
    at = ctypes.addressof
    run = lambda **over: _refused(api, "lrnnx_grad_clip", _fill(api.GradClipArgs, **{**dict(count=3, grads=at(grads), numel=at(n), dtype=at(kind), norm=FAR * 4, max_norm=1.0, eps=0.0), **over}))
    other = dict(out=at(out), out_dtype=at(wide))
    assert not run() and not run(norm=BUF + 20) and not run(norm=FAR + 200) and not run(norm=BUF, **other) and not run(norm=FAR * 3 + 400, **other)
    assert run(norm=BUF) and run(norm=BUF + 16) and run(norm=FAR + 196) and run(norm=FAR * 2 + 16, **other) and run(norm=FAR * 3 + 396, **other)


def test_gradients_over_the_words(api):  # noqa: F811
    base = dict(T=100, V=1000, K=64, io_dtype=1, h=FAR, h_stride=64, weight=BUF, weight_stride=70, target=FAR * 2, lse=FAR * 3, dloss=FAR * 4, dloss_stride=1, dh=FAR * 5, dweight=FAR * 6,
                workspace=FAR * 7, workspace_bytes=1 << 40)
    run = lambda **over: _refused(api, "lrnnx_vocab_loss_bwd", _fill(api.VocabBwdArgs, **{**base, **over}))
    end = (999 * 70 + 64) * 2
    assert not run() and not run(dweight=BUF + end) and not run(dh=BUF - 100 * 64 * 2) and not run(dh=None, dweight=FAR * 5)
    assert run(dweight=BUF) and run(dweight=BUF + end - 2) and run(dh=BUF + 4) and run(dh=FAR * 6 + 1000) and run(dh=None, dweight=BUF)
