"""The rules that choose kernels and launch shapes of the int8 product (csrc/vnm_i8_rules.h), compiled for the host and compared
with what was measured on both sides; and what the compiler made of the 8-bit kernels."""

import os
import shutil
import subprocess

import pytest

from paper_2410_16135_amd import build
from tests.test_kernel_registers import _kernels_of

CSRC = os.path.join(build.PKG_DIR, "csrc")


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    """rule("f(1, 2)", ...) evaluates expressions on the rules and returns them as floats."""
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("g++ not found")
    tmp = tmp_path_factory.mktemp("rules")

    def run(*exprs):
        src = tmp / "rule.cpp"
        src.write_text('#include "vnm_i8_rules.h"\n#include <cstdio>\nusing namespace vnm;\nint main() {\n'
                       + "".join('std::printf("%%.6f\\n", (double)(%s));\n' % e for e in exprs) + "}\n")
        exe = str(tmp / "rule")
        res = subprocess.run([cxx, "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", exe], capture_output=True, text=True)
        assert res.returncode == 0, res.stderr
        return [float(v) for v in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    return run


def _shape(rule, T, out, inn, M):
    R64, S = -(-out // 64), -(-(-(-inn // M)) // 16)
    call = "i8_few_shape(%d, %d, %d, %d)" % (T, R64, S, M)
    return tuple(int(v) for v in rule(call + ".tiles", call + ".tokens", call + ".waves"))


# (tiles, tokens, waves) of the fastest shape measured, or one within a tenth of it; us of the others in the comments
@pytest.mark.parametrize("T,out,inn,M,shape", [
    (1, 4096, 4096, 5, (1, 4, 4)), (16, 4096, 4096, 5, (1, 16, 4)),          # four waves 5.3, eight 5.4; 6.5, 6.0
    (1, 4096, 11008, 5, (1, 4, 8)), (16, 4096, 11008, 5, (1, 16, 8)),        # four waves 8.3, eight 7.9; 11.1, 8.9
    (8, 176, 5416, 5, (1, 4, 4)), (25, 144, 2424, 4, (1, 4, 4)),             # one group of 16: 6.8, four 5.7; 5.0, 4.5
    (64, 4096, 4096, 5, (1, 32, 4)), (128, 4096, 4096, 5, (2, 32, 4)),       # at 16 tokens 8.4, 8.0; at 32 of one tile 11.1, 9.0
    (583, 685, 1296, 5, (2, 32, 4)), (71, 296, 1288, 8, (1, 16, 4)),         # at 16 7.8, 6.6; at 32 5.0, 4.3
])
def test_shapes(rule, T, out, inn, M, shape):
    assert _shape(rule, T, out, inn, M) == shape


# few-token kernel where it was the faster one; us of it and of staging with the product
@pytest.mark.parametrize("T,out,inn,M,few", [
    (128, 4096, 4096, 5, 1), (256, 4096, 4096, 5, 1), (700, 4096, 4096, 5, 0),             # 9.1 / 24, 13.4 / 24.3, 29 / 27.6
    (700, 4096, 11008, 5, 0), (4096, 4096, 11008, 5, 0), (700, 2304, 768, 8, 1),           # 64 / 49, - / 105, 10.0 / 13.5
    (2048, 2304, 768, 8, 0), (916, 592, 10744, 10, 1), (1320, 1424, 129, 8, 1),            # 18.4 / 14.5, 24.3 / 47, 10.2 / 15.2
    (2241, 6848, 256, 6, 0), (4847, 648, 6704, 4, 0)])                                     # 45 / 16.4, 76 / 47
def test_few_or_staged(rule, T, out, inn, M, few):
    assert rule("i8_takes_few(%d, %d, %d, %d, %d)" % (T, -(-out // 64), inn, -(-(-(-inn // M)) // 16), M)) == [few]


def test_up_to_128_tokens_need_no_workspace(rule):
    sizes = [(T, R, inn, M) for T in (1, 4, 33, 128) for R in (1, 64, 172) for inn in (64, 4096, 20000) for M in (4, 16)]
    assert all(rule(*("i8_takes_few(%d, %d, %d, %d, %d)" % (T, R, i, -(-(-(-i // M)) // 16), M) for T, R, i, M in sizes)))


def test_workgroups_of_eight_row_blocks(rule):
    # 4096 tokens x 64 row blocks: 256 workgroups; 2048: 128, which leave half of the compute units idle; less than 8 row blocks never
    assert rule("i8_staged_wide(32, 64)", "i8_staged_wide(16, 64)", "i8_staged_wide(1000, 7)", "i8_staged_wide(130, 8)") == [1, 0, 0, 1]


@pytest.mark.parametrize("kernel", ["spmm_i8_few_kernel", "spmm_i8_staged_kernel", "stage_q_kernel", "quantize_rows_kernel", "pack_i8_kernel"])
def test_kernels_use_no_scratch_memory(kernel, tmp_path):
    readelf = "/opt/rocm/llvm/bin/llvm-readelf"
    if not os.path.exists(readelf) or build.built_hash() != build.source_hash():
        pytest.skip("llvm-readelf or an up-to-date library not found")
    used = {k: v for k, v in _kernels_of(build.LIB_PATH, tmp_path, readelf).items() if kernel in k}
    assert used, "kernel not found in the library"
    assert {k: v for k, v in used.items() if v} == {}
