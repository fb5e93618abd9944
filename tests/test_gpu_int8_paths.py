"""The int8 product's kernels and operand layouts against each other and the plain form, bit for bit."""

import pytest
import torch

import paper_2410_16135_amd as vnm
from tests import int8_reference as ref
from tests.test_gpu_int8 import DEV, make, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", list(range(4, 17)))
@pytest.mark.parametrize("V", [32, 64, 128])
def test_product_every_pattern(V, M):
    # widths that end inside a K step and inside a block; three row blocks and a partial one
    out, inn = 3 * V + 5, 16 * M * 3 + M + 3
    for T in (3, 40, 140):
        c, q, sx, sw, bias, dense, Q, SX = make(out, inn, V, M, T, 1000 * V + M)
        got = vnm.vnm_spmm_i8(Q, SX, c, out_dtype=torch.float32, path=vnm.PATH_SMFMAC)
        assert same(got, ref.product(q, sx, dense, sw, None, "fp32")), T


@pytest.mark.parametrize("T", [1, 16, 48, 300])
def test_product_paths_and_strides_agree(T):
    c, q, sx, sw, bias, dense, Q, SX = make(300, 700, 64, 6, T, 11)
    want = ref.product(q, sx, dense, sw, bias, "fp16")
    B = torch.from_numpy(bias).to(DEV)
    for path in (vnm.PATH_AUTO, vnm.PATH_GENERIC, vnm.PATH_SMFMAC):
        assert same(vnm.vnm_spmm_i8(Q, SX, c, bias=B, path=path), want)
    # rows of Q further apart, and rows that the matrix-core kernels cannot read
    for ld, first in ((1024, 0), (720, 16), (701, 0), (777, 5)):
        buf = torch.full((T + 1, ld), -3, dtype=torch.int8, device=DEV)
        view = buf[:T, first:first + 700]
        view.copy_(Q)
        assert same(vnm.vnm_spmm_i8(view, SX, c, bias=B), want), (ld, first)
    # Y with other strides and alignments: what stands around it stays
    for dtype, ld, first in (("fp16", 304, 0), ("fp16", 311, 3), ("fp32", 301, 1), ("bf16", 320, 8)):
        buf = torch.full((T + 2, ld + 8), 42.0, dtype=ref.TYPES[dtype], device=DEV)
        view = buf[1:T + 1, first:first + 300]
        vnm.vnm_spmm_i8(Q, SX, c, bias=B, Y=view)
        assert same(view, ref.product(q, sx, dense, sw, bias, dtype)), (dtype, ld, first)
        view.fill_(42.0)
        assert bool((buf == 42.0).all())
