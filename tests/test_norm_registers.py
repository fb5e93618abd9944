"""What the compiler made of the norm kernels: which of them use scratch memory, and how much of it."""

import os
import re

import pytest

from paper_2410_16135_amd import build
from tests.test_kernel_registers import _kernels_of

BIASES, GATED, POSTED = 1, 2, 4                    # parts of a backward kernel (csrc/vnm_norm_backward.hip)


def allowed(backward, all_fp32, threads, octets, parts):
    """Bytes of scratch per thread, at most: the comments beside the launch rules name the same kernels."""
    if not backward:
        return 0 if octets == 1 else 316
    if octets == 2:
        return 864
    if threads == 1024:
        return 176 if parts & (GATED | POSTED) else 0
    if parts == POSTED and (threads == 512 or all_fp32 and threads > 64):
        return 88 if all_fp32 else 28
    return 0


def test_scratch_memory_of_the_norms(tmp_path):
    readelf = "/opt/rocm/llvm/bin/llvm-readelf"
    if not os.path.exists(readelf) or build.built_hash() != build.source_hash():
        pytest.skip("llvm-readelf or an up-to-date library not found")
    seen = {False: 0, True: 0}
    for name, used in _kernels_of(build.LIB_PATH, tmp_path, readelf).items():
        m = re.search(r"residual_norm(_backward)?_kernelI(f|DF16_|DF16b)(f|DF16_|DF16b|S\w*_)Li(\d+)ELi(\d+)E(?:Li(\d+)E)?", name)
        if not m:
            assert "residual_norm" not in name, name
            continue
        backward, fp32 = m.group(1) is not None, (m.group(2), m.group(3)) == ("f", "f")
        assert used <= allowed(backward, fp32, int(m.group(4)), int(m.group(5)), int(m.group(6) or 0)), name
        seen[backward] += 1
    # five pairs of types: six widths forward; five parts at five widths and all parts at the sixth backward
    assert seen == {False: 5 * 6, True: 5 * (4 * 5 + 6)}


@pytest.mark.parametrize("kernel", ["column_reduce_kernel", "quantize_long_kernel", "spmm_i8_triple_kernel"])
def test_others_use_none(kernel, tmp_path):
    readelf = "/opt/rocm/llvm/bin/llvm-readelf"
    if not os.path.exists(readelf) or build.built_hash() != build.source_hash():
        pytest.skip("llvm-readelf or an up-to-date library not found")
    used = {k: v for k, v in _kernels_of(build.LIB_PATH, tmp_path, readelf).items() if kernel in k}
    assert used and {k: v for k, v in used.items() if v} == {}
