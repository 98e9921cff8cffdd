"""The kernels of the gated delta rule and of the norms around a block keep what they need in registers, but for the forms named here (no GPU: read from the
built library's kernel metadata).  What a step spills it reloads through the queue of its loads ahead: 1.7 times the time in the float32 walk of many heads."""
import os
import re

import pytest

from paper_2602_08810_amd import build
from test_kernel_registers import READELF, _spills

# k_delta_scan<I/O, planes of an input, of the state chain, dk, wavefronts to 16 columns, saving, in float32, of a segment>
SCAN = [rf"k_delta_scanIfLi3ELi3ELi(128|64)ELi1ELb(0ELb0|1ELb1)ELb0E",        # float32, a wavefront to 16 columns
        r"k_delta_scanIfLi3ELi3ELi128ELi2ELb(0ELb0|1ELb1)ELb0E", r"k_delta_scanIfLi3ELi3ELi64ELi2ELb1ELb1ELb0E",
        r"k_delta_scanItLi1ELi[23]ELi128ELi1ELb[01]ELb[01]ELb0E"]                # bfloat16, dk > 64, a wavefront to 16 columns
ADJOINT = [r"k_delta_adjointILi3ELi3ELi128ELi[12]ELb1ELb0ELb0E"]                # float32, dk > 64, loads one chunk ahead
# k_block_norm<I/O, stream, elements a piece, pieces a thread, backward>
NORM = [r"k_block_normI(tt|ff)Li4ELi4ELb1E", r"k_block_normItfLi(8ELi2|4ELi4)ELb1E",                  # aligned, more than 4096 columns, backward
        r"k_block_normItfLi1ELi8ELb1E", r"k_block_normI(tt|tf|ff)Li1ELi(12|16)ELb1E", r"k_block_normItfLi1ELi16ELb0E"]


@pytest.mark.skipif(not os.path.exists(READELF), reason="no llvm-readelf")
def test_only_the_forms_named_spill(tmp_path):
    if not os.path.exists(build.LIB):
        pytest.skip("liblrnnx.so not built (run python -m paper_2602_08810_amd.build)")
    spills = {n: c for n, c in _spills(tmp_path).items() if re.search(r"\d+k_(delta|block_norm|norm_sums)", n)}
    for kernel, least in (("delta_prep", 14), ("delta_scan", 34), ("delta_join", 8), ("delta_adjoint", 40), ("delta_grads", 6), ("delta_step", 4), ("block_norm", 60)):
        assert sum(kernel in n for n in spills) >= least, kernel
    others = {n: c for n, c in spills.items() if c and not any(re.search(p, n) for p in SCAN + ADJOINT + NORM)}
    assert not others, others
