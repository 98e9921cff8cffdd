"""CPU checks of the C entry points of the gated delta rule and of the norms around a block: the binding's mirrors of their argument structs,
the size queries, and every refusal (all of it host code that runs before anything is launched)."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PAIRS = {"lrnnx_delta_fwd_args": "DeltaFwdArgs", "lrnnx_delta_bwd_args": "DeltaBwdArgs", "lrnnx_delta_step_args": "DeltaStepArgs",
         "lrnnx_norm_fwd_args": "NormFwdArgs", "lrnnx_norm_bwd_args": "NormBwdArgs"}
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
P = 1 << 20                                       # an address that nothing reads: every call below is refused


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


def _fill(cls, **over):
    a = cls()
    a.struct_size = ctypes.sizeof(cls)
    for n, v in over.items():
        setattr(a, n, v)
    return a


def _call(api, name, a):
    f = getattr(api.lib(), name)
    f.argtypes, f.restype = [ctypes.c_void_p], ctypes.c_size_t if name.endswith("_bytes") else ctypes.c_int
    return f(ctypes.byref(a))


SIZES = dict(B=2, Hk=2, Hv=4, dk=64, dv=64, io_dtype=1, gate_dtype=0, scale=0.1)
INPUTS = {**{n: P for n in ("q", "k", "v", "g", "beta")},
          **{f"{n}_stride_{x}": 4096 for n in ("q", "k", "v", "g", "beta") for x in "bh"}}
SEQ = {**SIZES, **INPUTS, "L": 100, **{f"{n}_stride_l": 512 for n in ("q", "k", "v", "g", "beta")}}
BAD_SIZES = [(dict(B=0), INVALID), (dict(Hk=0), INVALID), (dict(Hk=3), INVALID), (dict(dk=0), INVALID), (dict(dv=-1), INVALID),
             (dict(io_dtype=2), INVALID), (dict(gate_dtype=2), INVALID), (dict(io_dtype=0, gate_dtype=1), INVALID),
             (dict(dk=129), UNSUPPORTED), (dict(dv=257), UNSUPPORTED), (dict(B=65536), UNSUPPORTED), (dict(Hk=1, Hv=65536), UNSUPPORTED)]


@pytest.mark.parametrize("name,cls,extra", [
    ("lrnnx_gated_delta_fwd", "DeltaFwdArgs", dict(o=P, workspace=P, workspace_bytes=1)),
    ("lrnnx_gated_delta_bwd", "DeltaBwdArgs", {**{n: P for n in ("dout", "saved", "dq", "dkey", "dval", "dg", "dbeta", "workspace")},
                                              "saved_bytes": 1 << 40, "workspace_bytes": 1}),
])
def test_sequence_calls_refuse(api, name, cls, extra):
    cls = getattr(api, cls)
    base = {**SEQ, **extra}
    for over, code in BAD_SIZES + [(dict(L=0), INVALID), (dict(L=1 << 41), UNSUPPORTED), (dict(L=1 << 38), UNSUPPORTED)]:
        assert _call(api, name, _fill(cls, **{**base, **over})) == code, over
    for n in ("q", "k", "v", "g", "beta", *(x for x in extra if not x.endswith("bytes") and x not in ("workspace", "saved"))):
        assert _call(api, name, _fill(cls, **{**base, n: None})) == INVALID, n
        assert _call(api, name, _fill(cls, **{**base, n: P + 1})) == INVALID, n
    assert _call(api, name, _fill(cls, **{**base, "cu_seqlens": P + 4})) == INVALID
    assert _call(api, name, _fill(cls, **{**base, "workspace": P + 8})) == INVALID
    assert _call(api, name, _fill(cls, **base)) == WORKSPACE
    assert _call(api, name, _fill(cls, **{**base, "workspace": None, "workspace_bytes": 1 << 40})) == WORKSPACE
    a = _fill(cls, **base)
    a.struct_size -= 8
    assert _call(api, name, a) == INVALID
    assert _call(api, name + "_workspace_bytes", a) == 0
    if name.endswith("bwd"):
        assert _call(api, name, _fill(cls, **{**base, "saved_bytes": 1, "workspace_bytes": 1 << 40})) == WORKSPACE
        assert _call(api, name, _fill(cls, **{**base, "saved": None})) == INVALID


def test_sizes_of_scratch(api):
    fwd = lambda **over: _fill(api.DeltaFwdArgs, **{**SEQ, "o": P, **over})
    ws, sv = "lrnnx_gated_delta_fwd_workspace_bytes", "lrnnx_gated_delta_saved_bytes"
    plain = _call(api, ws, fwd())
    assert plain > 0
    assert _call(api, ws, fwd(q=P + 2)) >= plain + 2 * 100 * 2 * 64 * 2             # unaligned rows are copied
    assert _call(api, ws, fwd(io_dtype=0)) > _call(api, ws, fwd(q=P + 2))            # float32: three planes of q and k
    assert _call(api, ws, fwd(L=6400)) > 20 * plain
    slots = 2 * 2                                                                   # two sequences of 100 steps
    states, err = slots * 4 * 64 * 64 * 2, 2 * 200 * 4 * 64 * 2
    assert states + err < _call(api, sv, fwd()) < 3 * (states + err)
    packed = fwd(cu_seqlens=P)                                                      # 100 / 64 + 2 slots on one axis of 100 steps
    assert 0 < _call(api, sv, packed) < _call(api, sv, fwd())
    assert _call(api, sv, fwd(dk=500)) == 0


def test_step_refuses(api):
    base = {**SIZES, **INPUTS, "state": P, "o": P}
    cls = api.DeltaStepArgs
    for over, code in BAD_SIZES:
        assert _call(api, "lrnnx_gated_delta_step", _fill(cls, **{**base, **over})) == code, over
    for n in ("q", "k", "v", "g", "beta", "state", "o"):
        assert _call(api, "lrnnx_gated_delta_step", _fill(cls, **{**base, n: None})) == INVALID, n
        assert _call(api, "lrnnx_gated_delta_step", _fill(cls, **{**base, n: P + 1})) == INVALID, n


NORM = dict(M=4, D=96, groups=1, io_dtype=1, res_dtype=0, eps=1e-6, x=P, x_stride=96)


def test_norm_refuses(api):
    bad = [(dict(M=0), INVALID), (dict(D=0), INVALID), (dict(groups=5), INVALID), (dict(groups=0), INVALID), (dict(gate_act=2), INVALID),
           (dict(io_dtype=2), INVALID), (dict(io_dtype=0, res_dtype=1), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
           (dict(x=None), INVALID), (dict(x=P + 1), INVALID), (dict(D=8193), UNSUPPORTED), (dict(M=1 << 41), UNSUPPORTED)]
    f, b = "lrnnx_block_norm_fwd", "lrnnx_block_norm_bwd"
    for over, code in bad + [(dict(h=None), INVALID), (dict(pre_weight=P), INVALID), (dict(y=P), INVALID), (dict(h=P + 2), INVALID)]:
        assert _call(api, f, _fill(api.NormFwdArgs, **{**NORM, "h": P, **over})) == code, over
    base = {**NORM, "dh": P, "dx": P, "workspace": P, "workspace_bytes": 1}
    for over, code in bad + [(dict(dx=None), INVALID), (dict(dh=None), INVALID), (dict(dy=P), INVALID), (dict(dgate=P), INVALID),
                             (dict(dresidual=P), INVALID), (dict(dpost_weight=P), INVALID), (dict(dres_scale=P), INVALID),
                             (dict(dpre_weight=P), INVALID), (dict(workspace=P + 4), INVALID), (dict(), WORKSPACE), (dict(workspace=None), WORKSPACE)]:
        assert _call(api, b, _fill(api.NormBwdArgs, **{**base, **over})) == code, over
    q = api.lib().lrnnx_block_norm_bwd_workspace_bytes
    assert q(0, 96) == 0 and q(4, 8193) == 0 and 0 < q(4, 96) <= 4 * 3 * 96 * 4
