"""What the compiler makes of the direct loads to LDS (no GPU: assembly of a kernel compiled here): it does not take the register that they write for its own value still."""
import os
import re
import subprocess

import pytest

from paper_2602_08810_amd import build

KERNEL = r"""
#include "lds_load.hpp"
using namespace lrnnx;
__global__ void k(const uint32_t *src, uint32_t *out, u32x4 d, int n) {
    __shared__ uint32_t lds[8192];
    const auto r = __builtin_amdgcn_make_buffer_rsrc((void *)src, 0, n, 0x00020000);
    const auto to = (__attribute__((address_space(3))) void *)lds;
    uint32_t off[PIECES_];
    for (int i = 0; i < PIECES_; ++i) off[i] = threadIdx.x * 16 + 4096 * i;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, to, 4, threadIdx.x * 4, 0, 0, 0);
    load_lds<PIECES_, 1024>(4096, d, off);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, to, 4, threadIdx.x * 4, 0, 256, 0);
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    out[threadIdx.x] = lds[threadIdx.x] + lds[threadIdx.x + 64] + lds[threadIdx.x + 1024];
}
"""


@pytest.mark.parametrize("count", [1, 2, 4])
def test_m0_is_set_again(tmp_path, count):
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    src, out = tmp_path / "k.hip", tmp_path / "k.s"
    src.write_text(KERNEL)
    subprocess.run([build.HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "--offload-device-only", "-S", f"-DPIECES_={count}", "-I", os.path.join(build.HERE, "csrc"),
                    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-o", str(out), str(src)], check=True, capture_output=True)
    text = out.read_text()
    loads = [m.start() for m in re.finditer(r"buffer_load_dword .* lds", text)]
    assert len(loads) == 2 and len(re.findall(r"buffer_load_dwordx4 .* lds", text)) == count
    between = text[loads[0]:loads[1]]
    assert "s_mov_b32 m0" in between[between.index("ASMEND"):]
