"""vnm_spmm_i8 where its rule takes the many-token kernels: staging and product in one call, bit for bit against the plain form."""

import pytest
import torch

import paper_2410_16135_amd as vnm
from tests import int8_reference as ref
from tests.test_gpu_int8 import DEV, make, same

pytestmark = pytest.mark.gpu


def many(out, inn, V, M, T, seed):
    """A case of test_gpu_int8.make that the many-token kernels serve."""
    case = make(out, inn, V, M, T, seed)
    assert vnm.vnm_spmm_i8_workspace_bytes(T, case[0]) > 0
    return case


def test_no_workspace_for_rows_that_are_not_staged():
    """Rows that the matrix-core kernels cannot read go to the kernel on the triple, which needs none."""
    T, out, inn = 1100, 2100, 1405
    c, q, sx, sw, bias, dense, Q, SX = many(out, inn, 64, 11, T, 31)
    want = ref.product(q, sx, dense, sw, None, "fp16")
    Y = torch.empty(T, out, dtype=torch.float16, device=DEV)

    def peak(x):
        before = torch.cuda.memory_allocated()
        torch.cuda.reset_peak_memory_stats()
        assert same(vnm.vnm_spmm_i8(x, SX, c, Y=Y), want)
        return torch.cuda.max_memory_allocated() - before

    assert peak(Q) >= vnm.vnm_spmm_i8_workspace_bytes(T, c)
    for ld, first in ((1405, 0), (1424, 8)):
        view = torch.zeros(T * ld + 16, dtype=torch.int8, device=DEV).as_strided((T, inn), (ld, 1), first)
        view.copy_(Q)
        assert peak(view) == 0, (ld, first)
