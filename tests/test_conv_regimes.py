"""CPU check that the calls of the convolution's tests against 64 bits run its main loops: the plans that the library makes for them."""
import os
import shutil
import subprocess

import pytest

from _conv_regimes import CASES
from paper_2602_08810_amd import build

PLAN = r"""
#include "conv.hpp"
#include <cstdio>
#include <cstdlib>
using namespace lrnnx;
int main(int, char **v) {
    static int64_t some;
    for (int backward = 0; backward < 2; ++backward) {
        ConvParams p{};
        p.time_last = atoi(v[1]); p.cu = atoi(v[2]) ? &some : nullptr; p.seqs = atoi(v[3]); p.B = p.cu ? 1 : p.seqs;
        p.L = atoll(v[4]); p.D = atoi(v[5]); p.W = atoi(v[6]); p.io = atoi(v[7]);
        plan_conv(p, backward);
        printf("%d %d %d %lld\n", p.blocks, p.tile, p.shift, (long long)p.tiles);
    }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if not os.path.exists(build.LIB) or not shutil.which("g++"):
        pytest.skip("liblrnnx.so not built, or no g++")
    d = tmp_path_factory.mktemp("plan")
    src, exe = d / "plan.cpp", d / "plan"
    src.write_text(PLAN)
    rocm = os.path.dirname(os.path.dirname(build.HIPCC))
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", f"-I{rocm}/include", "-I", os.path.join(build.HERE, "csrc"), str(src), "-o", str(exe), build.LIB,
                    f"-Wl,-rpath,{build.HERE}", f"-Wl,-rpath,{rocm}/lib", f"-L{rocm}/lib", "-lamdhip64"], check=True, capture_output=True)
    def run(*args):
        out = subprocess.run([str(exe), *(str(int(a)) for a in args)], check=True, capture_output=True, text=True).stdout
        return [tuple(int(x) for x in line.split()) for line in out.splitlines()]
    return run


@pytest.mark.parametrize("layout,B,L,D,W,io,packed,reaches", CASES)
def test_plans(plan, layout, B, L, D, W, io, packed, reaches):
    (_, tile, shift, _), (blocks, back, back_shift, tiles) = plan(layout == "bdl", packed, B, L, D, W, io == "bf16")
    piece = 8 if io == "bf16" else 4
    got = set()
    if layout == "bld":
        if back >= 16:
            got.add("inside")
        if tiles > blocks * (256 >> back_shift):
            got.add("turns")
    else:
        if back > (2 * piece << back_shift):
            got.add("visits")
        if tiles > blocks:
            got.add("turns")
        if tile > piece << shift:
            got.add("pieces")
    assert got >= reaches, (got, tile, shift, blocks, back, back_shift, tiles)
