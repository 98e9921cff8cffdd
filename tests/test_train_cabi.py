"""CPU checks of the C entry points of the short causal convolution, the loss over a vocabulary, and the norm and clipping of gradients: the binding's mirrors of
their argument structs, the size queries, and every refusal (all of it host code that runs before anything is launched)."""
import ctypes
import os
import re
import subprocess

import pytest

from test_delta_cabi import INVALID, P, ROOT, UNSUPPORTED, WORKSPACE, _call, _fill

PAIRS = {"lrnnx_conv_fwd_args": "ConvFwdArgs", "lrnnx_conv_bwd_args": "ConvBwdArgs", "lrnnx_conv_step_args": "ConvStepArgs",
         "lrnnx_vocab_fwd_args": "VocabFwdArgs", "lrnnx_vocab_bwd_args": "VocabBwdArgs", "lrnnx_grad_norm_args": "GradNormArgs",
         "lrnnx_grad_clip_args": "GradClipArgs"}


@pytest.fixture(scope="module")
def api():
    pytest.importorskip("torch")
    from paper_2602_08810_amd import api as _api, build
    if not os.path.exists(build.LIB):
        pytest.skip("liblrnnx.so not built (run python -m paper_2602_08810_amd.build)")
    return _api


def test_mirrors_have_the_header_s_layout(api, tmp_path):
    lines = ['#include <stdio.h>', '#include <stddef.h>', f'#include "{ROOT}/include/lrnnx.h"', "int main(void) {"]
    for cname, pyname in PAIRS.items():
        lines.append(f'  printf("{cname} %zu\\n", sizeof({cname}));')
        lines += [f'  printf("{cname}.{f} %zu\\n", offsetof({cname}, {f}));' for f, _ in getattr(api, pyname)._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["  return 0;", "}"]))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-o", str(exe), str(src)], check=True)
    got = dict(line.split() for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines())
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "lrnnx.h")).read(), flags=re.S)
    for cname, pyname in PAIRS.items():
        cls = getattr(api, pyname)
        assert int(got[cname]) == ctypes.sizeof(cls)
        for f, _ in cls._fields_:
            assert int(got[f"{cname}.{f}"]) == getattr(cls, f).offset, f
        body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (cname, cname), text, flags=re.S).group(1)
        names = [re.findall(r"[A-Za-z_][A-Za-z_0-9]*", part)[-1] for decl in body.split(";") if decl.strip() for part in decl.split(",")]
        assert names == [f for f, _ in cls._fields_]


CONV = dict(B=2, D=96, W=4, time_last=0, act=0, io_dtype=1, L=100, x=P, x_stride_b=9600, x_stride_s=96, weight=P)
BAD_CONV = [(dict(B=0), INVALID), (dict(D=0), INVALID), (dict(W=0), INVALID), (dict(act=2), INVALID), (dict(io_dtype=2), INVALID), (dict(x=None), INVALID),
            (dict(x=P + 1), INVALID), (dict(weight=None), INVALID), (dict(weight=P + 2), INVALID), (dict(bias=P + 2), INVALID), (dict(W=1), UNSUPPORTED),
            (dict(W=5), UNSUPPORTED), (dict(D=65537), UNSUPPORTED), (dict(B=65536), UNSUPPORTED)]
BAD_SEQ = [(dict(L=0), INVALID), (dict(time_last=2), INVALID), (dict(x0=P + 1), INVALID), (dict(cu_seqlens=P + 4), INVALID), (dict(L=(1 << 31) + 1), UNSUPPORTED)]


def test_convolution_refuses(api):
    f, b, s = "lrnnx_short_conv_fwd", "lrnnx_short_conv_bwd", "lrnnx_short_conv_step"
    for over, code in BAD_CONV + BAD_SEQ + [(dict(y=None), INVALID), (dict(y=P + 1), INVALID), (dict(x_last=P + 1), INVALID)]:
        assert _call(api, f, _fill(api.ConvFwdArgs, **{**CONV, "y": P, **over})) == code, over
    base = {**CONV, "dy": P, "dx": P, "dweight": P, "workspace": P, "workspace_bytes": 1}
    for over, code in BAD_CONV + BAD_SEQ + [(dict(dy=None), INVALID), (dict(dx=None), INVALID), (dict(dweight=None), INVALID), (dict(dbias=P), INVALID), (dict(dy=P + 1), INVALID),
                                            (dict(dx=P + 1), INVALID), (dict(dx_last=P + 1), INVALID), (dict(dx0=P + 1), INVALID), (dict(dweight=P + 2), INVALID),
                                            (dict(workspace=P + 8), INVALID), (dict(), WORKSPACE), (dict(workspace=None, workspace_bytes=1 << 40), WORKSPACE)]:
        assert _call(api, b, _fill(api.ConvBwdArgs, **{**base, **over})) == code, over
    step = {n: v for n, v in CONV.items() if n in ("B", "D", "W", "act", "io_dtype", "x", "x_stride_b", "weight")}
    for over, code in BAD_CONV + [(dict(state=None), INVALID), (dict(state=P + 1), INVALID), (dict(y=None), INVALID), (dict(y=P + 1), INVALID)]:
        assert _call(api, s, _fill(api.ConvStepArgs, **{**step, "state": P, "y": P, **over})) == code, over
    for name, cls in ((f, api.ConvFwdArgs), (b, api.ConvBwdArgs), (s, api.ConvStepArgs)):
        a = _fill(cls, **{n: v for n, v in CONV.items() if hasattr(cls, n)})
        a.struct_size += 8
        assert _call(api, name, a) == INVALID


@pytest.mark.parametrize("time_last", [0, 1])
@pytest.mark.parametrize("B,L,D", [(1, 1, 1), (1, 1, 65536), (8, 2048, 1536), (65535, 1, 1), (1, 1 << 32, 8), (65535, 65536, 65536), (3, 7, 9), (1, 100000, 64)])
def test_workspace_of_the_convolution_s_gradients(api, time_last, B, L, D):
    """Parts of W + 1 sums for every channel, no more of them than three workgroups a compute unit need."""
    a = _fill(api.ConvBwdArgs, **{**CONV, "B": B, "L": L, "D": D, "time_last": time_last})
    n = _call(api, "lrnnx_short_conv_bwd_workspace_bytes", a)
    assert n % (5 * D * 4) == 0 and 1 <= n // (5 * D * 4) <= 768
    a.W = 9
    assert _call(api, "lrnnx_short_conv_bwd_workspace_bytes", a) == 0


VOCAB = dict(T=100, V=1000, K=64, io_dtype=1, h=P, h_stride=64, weight=P, weight_stride=64, target=P)


def test_vocabulary_refuses(api):
    bad = [(dict(T=0), INVALID), (dict(V=0), INVALID), (dict(K=0), INVALID), (dict(io_dtype=2), INVALID), (dict(h=None), INVALID), (dict(weight=None), INVALID),
           (dict(target=None), INVALID), (dict(h=P + 1), INVALID), (dict(weight=P + 1), INVALID), (dict(target=P + 4), INVALID), (dict(T=(1 << 27) + 1), UNSUPPORTED),
           (dict(V=(1 << 27) + 1), UNSUPPORTED), (dict(K=(1 << 20) + 1), UNSUPPORTED), (dict(T=1 << 27, V=1 << 27), UNSUPPORTED)]
    fwd = {**VOCAB, "loss": P, "lse": P, "workspace": P, "workspace_bytes": 1}
    for over, code in bad + [(dict(loss=None), INVALID), (dict(lse=None), INVALID), (dict(loss=P + 2), INVALID), (dict(workspace=P + 16), INVALID), (dict(), WORKSPACE),
                             (dict(workspace=None), WORKSPACE)]:
        assert _call(api, "lrnnx_vocab_loss_fwd", _fill(api.VocabFwdArgs, **{**fwd, **over})) == code, over
    bwd = {**VOCAB, "lse": P, "dloss": P, "dh": P, "dweight": P, "workspace": P, "workspace_bytes": 1}
    for over, code in bad + [(dict(lse=None), INVALID), (dict(dloss=None), INVALID), (dict(dh=None, dweight=None), INVALID), (dict(dh=P + 1), INVALID), (dict(dweight=P + 1), INVALID),
                             (dict(dloss=P + 2), INVALID), (dict(workspace=P + 16), INVALID), (dict(), WORKSPACE), (dict(workspace=None), WORKSPACE)]:
        assert _call(api, "lrnnx_vocab_loss_bwd", _fill(api.VocabBwdArgs, **{**bwd, **over})) == code, over


def test_sizes_of_the_vocabulary_s_workspace(api):
    fwd = lambda **over: _call(api, "lrnnx_vocab_loss_fwd_workspace_bytes", _fill(api.VocabFwdArgs, **{**VOCAB, **over}))
    bwd = lambda **over: _call(api, "lrnnx_vocab_loss_bwd_workspace_bytes", _fill(api.VocabBwdArgs, **{**VOCAB, **over}))
    plain = fwd()
    assert 0 < plain < 100 * 1000 * 2                                                # not the logits
    assert fwd(h=P + 2) >= plain + 100 * 64 * 2 and fwd(weight_stride=65) >= plain + 1000 * 64 * 2       # copies
    assert plain + 3 * 100 * 64 * 2 <= fwd(io_dtype=0) < 3 * 1000 * 64 * 2            # few rows: of h alone
    assert fwd(io_dtype=0, T=600) >= plain + 3 * 1600 * 64 * 2
    assert bwd() >= 100 * 1000 * 2
    large = dict(T=1 << 15, V=1 << 18, K=4096, h_stride=4096, weight_stride=4096)
    assert bwd(**large) < (5 << 30)                                                  # 16 GB of logits: a piece of dz of 1 GiB and the parts of dh
    assert fwd(**{**large, "io_dtype": 0}) < (3 << 30)                               # a copied piece of the vocabulary
    assert fwd(K=0) == 0 and bwd(T=0) == 0


def test_gradients_refuse(api):
    n = (ctypes.c_int64 * 2)(5, 0)
    ptr = (ctypes.c_void_p * 2)(P, None)
    kind = (ctypes.c_int32 * 2)(0, 1)
    at = ctypes.addressof
    base = dict(count=2, grads=at(ptr), numel=at(n), dtype=at(kind), norm=P)
    neg, odd, none, unknown = (ctypes.c_int64 * 2)(5, -1), (ctypes.c_void_p * 2)(P + 2, None), (ctypes.c_void_p * 2)(None, None), (ctypes.c_int32 * 2)(0, 2)
    huge = (ctypes.c_int64 * 2)(5, (1 << 44) + 1)
    bad = [(dict(count=0), INVALID), (dict(grads=None), INVALID), (dict(numel=None), INVALID), (dict(dtype=None), INVALID), (dict(norm=None), INVALID), (dict(norm=P + 2), INVALID),
           (dict(numel=at(neg)), INVALID), (dict(grads=at(odd)), INVALID), (dict(grads=at(none)), INVALID), (dict(dtype=at(unknown)), INVALID), (dict(numel=at(huge)), UNSUPPORTED)]
    for over, code in bad + [(dict(workspace=P + 4), INVALID), (dict(), WORKSPACE), (dict(workspace=P, workspace_bytes=4), WORKSPACE)]:
        assert _call(api, "lrnnx_grad_norm", _fill(api.GradNormArgs, **{**base, **over})) == code, over
    narrow = (ctypes.c_int32 * 2)(1, 1)
    clip = {**base, "max_norm": 1.0, "eps": 1e-6}
    for over, code in bad + [(dict(max_norm=-1.0), INVALID), (dict(max_norm=float("nan")), INVALID), (dict(eps=-1.0), INVALID), (dict(out=at(ptr)), INVALID),
                             (dict(out=at(ptr), out_dtype=at(narrow)), INVALID), (dict(out=at(none), out_dtype=at(kind)), INVALID), (dict(out=at(odd), out_dtype=at(kind)), INVALID)]:
        assert _call(api, "lrnnx_grad_clip", _fill(api.GradClipArgs, **{**clip, **over})) == code, over

    def sizes(*v):
        numel = (ctypes.c_int64 * len(v))(*v)
        return _call(api, "lrnnx_grad_norm_workspace_bytes", _fill(api.GradNormArgs, count=len(v), numel=at(numel), grads=P, dtype=P, norm=P))
    assert sizes(0, 0) == 0 and sizes(5, -1) == 0 and sizes(1) == 8 and sizes(8192, 8193, 0) == 24
    # pieces of total / 16384 elements rounded up by less than 2048: at least 16384 / (1 + 2048 * 16384 / total) of them
    assert 16329 * 8 <= sizes(10 ** 10) <= 16384 * 8


def test_few_float32_rows_copy_no_vocabulary(api):
    """Whatever the start and step of its rows."""
    for name, cls, more in (("lrnnx_vocab_loss_fwd", api.VocabFwdArgs, {}), ("lrnnx_vocab_loss_bwd", api.VocabBwdArgs, dict(dloss=P, dh=P, dweight=P))):
        size = lambda **over: _call(api, name + "_workspace_bytes", _fill(cls, **{**VOCAB, "V": 50000, "K": 1001, "h_stride": 1001, "weight_stride": 1001, "io_dtype": 0, **more, **over}))
        assert 0 < size(T=20) < 50000 * 1001 * 2
        assert size(T=20, weight_stride=1003) == size(T=20, weight=P + 4) == size(T=20)
        assert size(T=20, weight_stride=0) >= size(T=20) + 50000 * 1001 * 4              # rows in one place are copied
