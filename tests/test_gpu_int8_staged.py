"""vnm_spmm_i8 where its rule takes the many-token kernels: staging and product in one call, bit for bit against the plain form."""

import numpy as np
import pytest
import torch

import paper_2410_16135_amd as vnm
import synth_inputs as syn
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


# --- every instantiation of the many-token loop -----------------------------------------------------------------------

def on_device(out, inn, V, M, T, seed):
    """As make, with activations and the plain product on the device (fp64, exact): layer, Q, scales, bias, fp32 sums."""
    rng = np.random.default_rng(seed)
    values, meta, col, sw, dense = ref.random_triple(rng, out, inn, V, M)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a).reshape(-1)).to(DEV)
    c = vnm.vnm_pack_i8(vnm.CompressedI8(dev(values), dev(meta), dev(col), None, dev(sw), out, inn, V, M))
    g = torch.Generator(device=DEV).manual_seed(seed)
    rows = torch.randint(-128, 128, (T, -(-inn // 16) * 16), generator=g, device=DEV, dtype=torch.int8)
    sx = torch.rand(T, generator=g, device=DEV) * 1e-1 + 1e-3
    bias = torch.randn(out, generator=g, device=DEV).half()
    Q = rows[:, :inn]
    sums = Q.double() @ torch.from_numpy(dense).to(DEV).double().t().contiguous()
    return c, Q, sx, bias, sums.float()


def plain(sums, sx, c, bias, dtype):
    y = (sums * c.scale[None]) * sx[:, None]
    return (y if bias is None else y + bias.float()[None]).to(dtype)


def form_of(T, out, inn, V, M):
    """(row blocks per workgroup, groups of waves on pieces of K) as csrc/vnm_i8_rules.h and vnm_spmm_i8_staged.hip choose them,
    and the K steps."""
    tiles, R, S = -(-T // 128), -(-(-(-out // V) * V) // 64), -(-(-(-inn // M)) // 16)
    if R >= 8 and tiles * -(-R // 8) > 128:
        return 8, 1, S
    rings = 160 // (2 * -(-16 * M * 144 // 1024))
    return 4, 2 if rings >= 3 and S >= 8 else 1, S


# K steps below, at and above the length of the rings (3 to 6 images) and of the rotations (5 or 6 sets of weights), odd and even
STEPS = [1, 2, 3, 4, 5, 6, 7, 8, 9, 11, 12, 13, 18, 23]


@pytest.mark.parametrize("M", list(range(4, 17)))
@pytest.mark.parametrize("V", [32, 64, 128])
def test_every_pattern_and_number_of_steps(V, M):
    """Eight row blocks, four on halves of K, and four, with one column table per row block and with two (V = 32)."""
    seen = set()
    for S in STEPS:
        for T, out in ((130, 5 * 64 + 9), (8300, 8 * 64 + 5)):
            inn = 16 * M * S - 5
            blocks, groups, steps = form_of(T, out, inn, V, M)
            assert steps == S and blocks == (8 if T > 4000 else 4)
            seen.add((blocks, groups))
            c, Q, sx, bias, sums = on_device(out, inn, V, M, T, 1000 * M + S)
            dtype = (torch.float16, torch.bfloat16, torch.float32)[S % 3]
            want = plain(sums, sx, c, bias, dtype)
            staged = vnm.vnm_stage_q(Q, M)
            assert torch.equal(vnm.vnm_spmm_i8_staged(staged, sx, c, bias=bias, out_dtype=dtype), want), (S, T)
            assert torch.equal(vnm.vnm_spmm_i8(Q, sx, c, bias=bias, out_dtype=dtype, path=vnm.PATH_SMFMAC), want), (S, T)
    assert seen == ({(8, 1), (4, 1), (4, 2)} if M <= 11 else {(8, 1), (4, 1)})


@pytest.mark.parametrize("T,out,inn,V,M,blocks,groups", [
    (700, 4100, 509, 64, 4, 4, 2), (700, 4096, 4096, 32, 6, 4, 2), (1100, 2100, 1405, 128, 11, 4, 2), (2048, 4096, 4096, 64, 5, 4, 2),
    (1576, 2304, 768, 128, 8, 4, 1), (4200, 1000, 1400, 64, 12, 4, 1), (4200, 1000, 253, 32, 16, 4, 1),
    (4096, 4096, 4096, 64, 5, 8, 1), (4096, 4096, 1100, 32, 7, 8, 1), (8400, 520, 1153, 128, 9, 8, 1), (8400, 520, 4000, 32, 16, 8, 1)])
def test_one_call(T, out, inn, V, M, blocks, groups):
    """Staging and product in one call, with and without a bias, for all result types."""
    assert form_of(T, out, inn, V, M)[:2] == (blocks, groups)
    c, Q, sx, bias, sums = on_device(out, inn, V, M, T, T + M)
    assert vnm.vnm_spmm_i8_workspace_bytes(T, c) > 0
    for dtype, b in ((torch.float16, bias), (torch.bfloat16, None), (torch.float32, bias)):
        assert torch.equal(vnm.vnm_spmm_i8(Q, sx, c, bias=b, out_dtype=dtype), plain(sums, sx, c, b, dtype)), dtype


def test_workspace():
    """One that is too small is refused; one of the right size may hold anything before the call, and nothing behind it is written."""
    T = 1100
    c, Q, sx, bias, sums = on_device(2100, 1405, 64, 11, T, 4)
    need = vnm.vnm_spmm_i8_workspace_bytes(T, c)
    assert need > 0
    with pytest.raises(vnm.VnmError, match="workspace"):
        vnm.vnm_spmm_i8(Q, sx, c, workspace=torch.empty(need - 1, dtype=torch.uint8, device=DEV))
    want = plain(sums, sx, c, None, torch.float16)
    for fill in (0, 0x80, 0xff):
        ws = torch.full((need + 4096,), fill, dtype=torch.uint8, device=DEV)
        assert torch.equal(vnm.vnm_spmm_i8(Q, sx, c, workspace=ws[:need]), want)
        assert bool((ws[need:] == fill).all())


@pytest.mark.parametrize("T,out,inn,V,M", [(1100, 2100, 1405, 64, 11), (700, 4096, 4096, 32, 6), (4200, 1000, 1400, 64, 12), (8400, 520, 1153, 64, 9)])
def test_on_streams_and_in_graphs(T, out, inn, V, M):
    """Staging buffers from the allocator of each stream and of each graph: two streams at once, two graphs in turn with eager
    calls between, other inputs every time."""
    c, Q, sx, bias, sums = on_device(out, inn, V, M, T, 21)
    assert vnm.vnm_spmm_i8_workspace_bytes(T, c) > 0
    inputs = [(Q, plain(sums, sx, c, bias, torch.float16))]
    inputs.append((Q.flip(0).contiguous() if inn % 16 == 0 else Q.new_zeros(T, -(-inn // 16) * 16)[:, :inn].copy_(Q.flip(0)),
                   plain(sums.flip(0), sx, c, bias, torch.float16)))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for k in range(8):
        with torch.cuda.stream(streams[k % 2]):
            got.append(vnm.vnm_spmm_i8(inputs[k % 2][0], sx, c, bias=bias))
    torch.cuda.synchronize()
    assert all(torch.equal(g, inputs[k % 2][1]) for k, g in enumerate(got))
    held = Q.new_zeros(T, -(-inn // 16) * 16)[:, :inn]
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = vnm.vnm_spmm_i8(held, sx, c, bias=bias)
        graphs.append((g, y))
    for k in range(4):
        held.copy_(inputs[k % 2][0])
        for g, y in graphs:
            y.zero_()
            g.replay()
        eager = vnm.vnm_spmm_i8(held, sx, c, bias=bias)
        torch.cuda.synchronize()
        assert torch.equal(eager, inputs[k % 2][1]) and all(torch.equal(y, inputs[k % 2][1]) for _, y in graphs)


# --- few tokens on long rows ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("M", list(range(4, 17)))
@pytest.mark.parametrize("V", [32, 64, 128])
def test_few_tokens_on_long_rows(V, M):
    """Eight waves cut K where it has 96 steps or more and there are at most 64 row blocks: groups of 4, 16 and 32 tokens."""
    for S, out, tokens in ((96, 130, (1, 3, 4, 5, 17, 33, 70)), (101, 2112, (9, 16, 17, 31, 32, 64))):
        inn = 16 * M * S - 5
        assert 2 * -(-(-(-out // V) * V) // 64) <= 128
        c, Q, sx, bias, sums = on_device(out, inn, V, M, max(tokens), 7 * M + V)
        for T in tokens:
            assert vnm.vnm_spmm_i8_workspace_bytes(T, c) == 0
            y = vnm.vnm_spmm_i8(Q[:T], sx[:T], c, bias=bias, path=vnm.PATH_SMFMAC)
            assert torch.equal(y, plain(sums[:T], sx[:T], c, bias, torch.float16)), (S, T)


# --- the packed copy --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("out,inn,V,M", [(128, 128, 64, 8), (130, 200, 32, 5), (384, 1536, 128, 16), (70, 37, 64, 6)])
def test_quantizing_a_layer_packs_it_as_packing_does(out, inn, V, M):
    """Every byte that the two calls write, into memory that was filled before."""
    W, _ = syn.make_weight_and_input(out, inn, 1, seed=out + M)
    f = vnm.vnm_prune_compress(torch.from_numpy(W).to(DEV), V, M)
    q = vnm.vnm_quantize_compressed(f)
    lib, stream = vnm.load_library(), torch.cuda.current_stream().cuda_stream
    for fill in (0, 0xa5):
        mine = torch.full_like(q.packed, fill)
        values, scale = torch.empty_like(q.values), torch.empty_like(q.scale)
        assert lib.vnm_quantize_compressed(f.values.data_ptr(), f.meta.data_ptr(), f.colidx.data_ptr(), out, inn, V, 2, M, values.data_ptr(),
                                           scale.data_ptr(), mine.data_ptr(), stream) == 0
        again = vnm.vnm_pack_i8(vnm.CompressedI8(q.values, q.meta, q.colidx, torch.full_like(q.packed, fill), q.scale, out, inn, V, M))
        assert torch.equal(values, q.values) and torch.equal(scale, q.scale) and torch.equal(mine, again.packed)
        assert not bool((mine == fill).all())
    # and the layer that the binding left multiplies as the one packed again does
    x, s = vnm.vnm_quantize_x(torch.randn(9, inn, device=DEV))
    assert torch.equal(vnm.vnm_spmm_i8(x, s, q), vnm.vnm_spmm_i8(x, s, again))
