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


@pytest.mark.parametrize("T", [1, 63, 128, 129, 700])
@pytest.mark.parametrize("inn,M", [(128, 4), (333, 5), (1030, 8), (600, 16)])
def test_shared_staging(inn, M, T):
    """Two layers of other widths, row blocks, types and biases on activations that are staged once."""
    staged = None
    for out, V, dtype in ((70, 64, "fp16"), (600, 32, "bf16"), (130, 128, "fp32")):
        c, q, sx, sw, bias, dense, Q, SX = make(out, inn, V, M, T, 17)
        if staged is None:
            first, staged = (q, sx, SX), vnm.vnm_stage_q(Q, M)
        b = bias if V != 32 else None
        got = vnm.vnm_spmm_i8_staged(staged, first[2], c, bias=None if b is None else torch.from_numpy(b).to(DEV), out_dtype=ref.TYPES[dtype])
        assert same(got, ref.product(first[0], first[1], dense, sw, b, dtype)), (out, V)


def test_shared_staging_buffer_too_small():
    c, q, sx, sw, bias, dense, Q, SX = make(128, 256, 64, 8, 200, 3)
    staged = vnm.vnm_stage_q(Q, 8)
    for call in (lambda: vnm.vnm_stage_q(Q, 8, staged=staged[:-256]), lambda: vnm.vnm_spmm_i8_staged(staged[:-256], SX, c)):
        with pytest.raises(vnm.VnmError, match="workspace"):
            call()


def test_staging_reads_no_row_past_the_last():
    """The activations end with their storage: rows of 16-byte pieces of which the last is cut."""
    T, inn = 150, 1000 - 3
    c, q, sx, sw, bias, dense, Q, SX = make(192, inn, 64, 5, T, 23)
    buf = torch.zeros((T - 1) * 1008 + inn + 11, dtype=torch.int8, device=DEV)        # (up to the piece's end)
    view = buf[:(T - 1) * 1008 + inn].as_strided((T, inn), (1008, 1))
    view.copy_(Q)
    want = ref.product(q, sx, dense, sw, None, "fp16")
    assert same(vnm.vnm_spmm_i8(view, SX, c), want)
    assert same(vnm.vnm_spmm_i8_staged(vnm.vnm_stage_q(view, 5), SX, c), want)


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("out,inn,V,M,T", [(203, 600, 64, 4, 193), (130, 100, 32, 8, 140), (602, 64, 128, 4, 8300)])
def test_stores_of_any_alignment(out, inn, V, M, T, dtype):
    """Two groups of waves on halves of K, one group, and eight row blocks: rows of Y that allow stores of 16 bytes, of 4, of one
    value; the values around Y stay."""
    c, q, sx, sw, bias, dense, Q, SX = make(out, inn, V, M, T, out + T)
    staged, b = vnm.vnm_stage_q(Q, M), torch.from_numpy(bias).to(DEV)
    want = ref.product(q, sx, dense, sw, bias, dtype)
    for first, ld in ((0, 608), (2, 608), (1, 608), (0, 606), (4, 604), (0, 605)):
        buf = torch.full((T + 2, ld + 8), 42.0, dtype=ref.TYPES[dtype], device=DEV)
        view = buf.as_strided((T, out), (ld, 1), ld + 3 - (ld + 3) % 8 + first)
        vnm.vnm_spmm_i8_staged(staged, SX, c, bias=b, Y=view)
        assert same(view, want), (first, ld)
        view.fill_(42.0)
        assert bool((buf == 42.0).all())
