"""The kernels of the short causal convolution, the loss over a vocabulary and the clipping of gradients keep what they need in registers (no GPU: read from the built
library's kernel metadata), but for the forms named here."""
import os
import re

import pytest

from paper_2602_08810_amd import build
from test_kernel_registers import READELF, _spills

# k_conv_rows_bwd<I/O, W, elements a piece, silu>: at most 168 registers, so that a compute unit has three workgroups
SPILLING = [r"k_conv_rows_bwdItLi[34]ELi4E"]


@pytest.mark.skipif(not os.path.exists(READELF), reason="no llvm-readelf")
def test_only_the_forms_named_spill(tmp_path):
    if not os.path.exists(build.LIB):
        pytest.skip("liblrnnx.so not built (run python -m paper_2602_08810_amd.build)")
    spills = {n: c for n, c in _spills(tmp_path).items() if re.search(r"\d+k_(conv|vocab|grad)_", n)}
    for kernel, least in (("conv_rows_fwd", 24), ("conv_rows_bwd", 24), ("conv_time_fwd", 24), ("conv_time_bwd", 24), ("conv_step", 12), ("conv_sums", 1), ("vocab_logits", 6),
                          ("vocab_dh", 3), ("vocab_dw", 3), ("vocab_pack", 2), ("vocab_add", 4), ("grad_squares", 1), ("grad_total", 1), ("grad_scale", 1)):
        assert sum(kernel in n for n in spills) >= least, kernel
    others = {n: c for n, c in spills.items() if c and not any(re.search(p, n) for p in SPILLING)}
    assert not others, others
