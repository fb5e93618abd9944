"""The 8-bit layer on the GPU: int8 activations and the int8 product against their plain forms, bit for bit (sums are exact in
int32 and every later operation is a single fp32 rounding), and a run of quantizer, product and norms together."""

import numpy as np
import pytest
import torch

import paper_2410_16135_amd as vnm
import synth_inputs as syn
from oracle import vnm_oracle as orc
from tests import int8_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def bits(t):
    return t.contiguous().view({2: torch.int16, 4: torch.int32}[t.element_size()]).cpu()


def same(got, want):
    """Equal bits; NaN equals NaN."""
    got, want = got.cpu(), want.cpu()
    return got.dtype == want.dtype and bool(((bits(got) == bits(want)) | (torch.isnan(got) & torch.isnan(want))).all())


# --- activations ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("T,n", [(1, 1), (3, 7), (5, 64), (33, 512), (2, 513), (7, 1000), (4, 2047), (9, 4096), (3, 4104), (2, 8191),
                                 (3, 11008), (2, 16384), (2, 16385), (1, 40000)])
def test_quantize(T, n, dtype):
    rng = np.random.default_rng(T * 100003 + n)
    x = torch.from_numpy(rng.standard_normal((T, n), dtype=np.float32) * np.exp(rng.uniform(-8, 8, (T, 1)))).to(ref.TYPES[dtype])
    if T > 2:
        x[0] = 0
        x[1, n // 2] = float("nan") if n % 2 else float("inf")
    want_q, want_s = ref.quantize_rows(x.float().numpy())
    q, s = vnm.vnm_quantize_x(x.to(DEV))
    assert np.array_equal(q.cpu().numpy(), want_q)
    assert same(s, torch.from_numpy(want_s))


def test_quantize_halves_and_extremes():
    # 127 / 127 = 1: values that lie half way between two integers go to the even one; the smallest and the largest fp32 rows
    x = np.zeros((6, 64), np.float32)
    x[0, :6] = [127, 0.5, 1.5, -2.5, 126.5, -0.49999997]
    x[1, :2] = [2.0 ** -100, -(2.0 ** -101)]
    x[2, :2] = [2.0 ** -101, 2.0 ** -140]
    x[3, :2] = [3.4e38, -1.7e38]
    x[4, :2] = [-0.0, 0.0]
    x[5, 63] = -np.inf
    want_q, want_s = ref.quantize_rows(x)
    q, s = vnm.vnm_quantize_x(torch.from_numpy(x).to(DEV))
    assert np.array_equal(q.cpu().numpy(), want_q) and same(s, torch.from_numpy(want_s))
    assert want_q[0, :6].tolist() == [127, 0, 2, -2, 126, 0]


def test_quantize_leaves_the_rest_of_the_rows():
    x = torch.randn(5, 40, dtype=torch.float16, device=DEV)[:, 3:30]           # 27 channels, unaligned rows
    buf = torch.full((7, 50), 99, dtype=torch.int8, device=DEV)
    scale = torch.full((7,), 5.0, device=DEV)
    vnm.vnm_quantize_x(x, Q=buf[1:6, 2:29], scale=scale[1:6])
    want_q, want_s = ref.quantize_rows(x.float().cpu().numpy())
    assert np.array_equal(buf[1:6, 2:29].cpu().numpy(), want_q) and same(scale[1:6], torch.from_numpy(want_s))
    rest = buf.clone()
    rest[1:6, 2:29] = 99
    assert bool((rest == 99).all()) and scale[0] == 5 and scale[6] == 5


def test_quantize_no_tokens():
    q, s = vnm.vnm_quantize_x(torch.empty(0, 64, dtype=torch.float16, device=DEV))
    assert q.shape == (0, 64) and s.shape == (0,)


# --- weights ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("out,inn,V,M", [(128, 128, 64, 8), (100, 37, 16, 6), (130, 200, 32, 5), (384, 1536, 128, 16), (70, 600, 64, 20)])
def test_quantize_compressed(out, inn, V, M):
    W, _ = syn.make_weight_and_input(out, inn, 1, seed=out + M)
    W[3] = 0                                                                    # a channel without weights
    c = vnm.vnm_prune_compress(torch.from_numpy(W).to(DEV), V, M)
    q = vnm.vnm_quantize_compressed(c)
    values = c.values.cpu().numpy().reshape(-1, 2 * -(-inn // M)).astype(np.float32)
    want_q, want_s = ref.quantize_rows(values)
    assert np.array_equal(q.values.cpu().numpy().reshape(want_q.shape), want_q)
    assert np.array_equal(q.scale.cpu().numpy(), want_s[:out]) and want_s[3] == 0
    if q.packed is not None:
        # the packed copy of both calls is the same in every byte that a kernel uses (the rest is slack)
        again = vnm.vnm_pack_i8(vnm.CompressedI8(q.values, q.meta, q.colidx, torch.zeros_like(q.packed), q.scale, out, inn, V, M))
        first = vnm.vnm_pack_i8(vnm.CompressedI8(q.values, q.meta, q.colidx, torch.zeros_like(q.packed), q.scale, out, inn, V, M))
        assert torch.equal(again.packed, first.packed)
    else:
        assert V == 16 or M > 16


# --- product ----------------------------------------------------------------------------------------------------------

def make(out, inn, V, M, T, seed, packed=True):
    rng = np.random.default_rng(seed)
    values, meta, col, sw, dense = ref.random_triple(rng, out, inn, V, M)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a).reshape(-1)).to(DEV)
    c = vnm.CompressedI8(dev(values), dev(meta), dev(col), None, dev(sw), out, inn, V, M)
    if packed:
        vnm.vnm_pack_i8(c)
    q = rng.integers(-128, 128, (T, inn)).astype(np.int8)
    sx = rng.uniform(1e-3, 1e-1, T).astype(np.float32)
    bias = rng.standard_normal(out).astype(np.float16)
    rows = torch.full((T, -(-inn // 16) * 16), 77, dtype=torch.int8, device=DEV)   # what stands behind a row is not read as a value
    rows[:, :inn] = torch.from_numpy(q).to(DEV)
    return c, q, sx, sw, bias, dense, rows[:, :inn], torch.from_numpy(sx).to(DEV)


TOKENS = [1, 2, 5, 16, 17, 31, 32, 33, 64, 65, 100, 128, 129, 200, 257]


@pytest.mark.parametrize("T", TOKENS)
@pytest.mark.parametrize("out,inn,V,M", [(64, 64, 64, 4), (128, 128, 64, 8), (200, 333, 32, 5), (100, 200, 128, 7), (192, 1030, 64, 16)])
def test_product_bits(out, inn, V, M, T):
    c, q, sx, sw, bias, dense, Q, SX = make(out, inn, V, M, T, T + 7 * out)
    for dtype in ("fp16", "bf16", "fp32"):
        b = bias if dtype != "bf16" else None
        want = ref.product(q, sx, dense, sw, b, dtype)
        got = vnm.vnm_spmm_i8(Q, SX, c, bias=None if b is None else torch.from_numpy(b).to(DEV), out_dtype=ref.TYPES[dtype])
        assert same(got, want), dtype


@pytest.mark.parametrize("out,inn,V,M,T", [(50, 37, 16, 6, 9), (100, 600, 64, 20, 5), (33, 255, 128, 255, 3), (1, 1, 16, 4, 1), (64, 5, 64, 16, 2),
                                           (64, 64, 64, 4, 70000)])
def test_product_without_a_packed_copy(out, inn, V, M, T):
    c, q, sx, sw, bias, dense, Q, SX = make(out, inn, V, M, T, 5, packed=False)
    got = vnm.vnm_spmm_i8(Q, SX, c, bias=torch.from_numpy(bias).to(DEV), out_dtype=torch.float32)
    assert same(got, ref.product(q, sx, dense, sw, bias, "fp32"))


@pytest.mark.parametrize("out,inn,V,M,T", [(2048, 1024, 64, 5, 1), (1000, 4096, 64, 8, 16), (1152, 384, 64, 5, 1576), (512, 4100, 32, 6, 700),
                                           (4096, 512, 128, 5, 300), (640, 11008, 64, 5, 500), (320, 768, 64, 16, 2100)])
def test_product_larger(out, inn, V, M, T):
    c, q, sx, sw, bias, dense, Q, SX = make(out, inn, V, M, T, 9)
    got = vnm.vnm_spmm_i8(Q, SX, c, bias=torch.from_numpy(bias).to(DEV))
    assert same(got, ref.product(q, sx, dense, sw, bias, "fp16"))


def test_product_largest_sums():
    # every product 128 * 128, as many as the layer has: the largest int32 sum of the width
    out, inn, V, M, T = 64, 4096, 64, 4, 3
    c, q, sx, sw, bias, dense, Q, SX = make(out, inn, V, M, T, 2, packed=False)
    c.values.fill_(-128)
    c.scale.fill_(1.0)
    vnm.vnm_pack_i8(c)
    for fill, n in ((-128, 16384), (127, -16256)):
        Q.fill_(fill)
        got = vnm.vnm_spmm_i8(Q, torch.ones(T, device=DEV), c, out_dtype=torch.float32)
        assert bool((got == float(n * 2 * (inn // M))).all())


def test_product_scales_that_are_not_numbers():
    c, q, sx, sw, bias, dense, Q, SX = make(128, 256, 64, 8, 20, 3)
    sx[3], sx[7], sx[9] = np.nan, np.inf, 0.0
    got = vnm.vnm_spmm_i8(Q, torch.from_numpy(sx).to(DEV), c, out_dtype=torch.float32)
    assert same(got, ref.product(q, sx, dense, sw, None, "fp32"))
    assert bool(torch.isnan(got[3]).all()) and not bool(torch.isnan(got[4]).any())


def test_product_results_beyond_fp16():
    c, q, sx, sw, bias, dense, Q, SX = make(128, 256, 64, 8, 20, 4)
    sx[:] = 1e6
    assert same(vnm.vnm_spmm_i8(Q, torch.from_numpy(sx).to(DEV), c), ref.product(q, sx, dense, sw, None, "fp16"))


def test_product_no_tokens():
    c, *_ = make(128, 256, 64, 8, 1, 4)
    y = vnm.vnm_spmm_i8(torch.empty(0, 256, dtype=torch.int8, device=DEV), torch.empty(0, device=DEV), c)
    assert y.shape == (0, 128)


def test_product_workspace_too_small():
    c, q, sx, sw, bias, dense, Q, SX = make(256, 512, 64, 8, 600, 4)
    need = vnm.vnm_spmm_i8_workspace_bytes(600, c)
    if need > 0:
        with pytest.raises(vnm.VnmError, match="workspace"):
            vnm.vnm_spmm_i8(Q, SX, c, workspace=torch.empty(need - 1, dtype=torch.uint8, device=DEV))
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    assert same(vnm.vnm_spmm_i8(Q, SX, c, workspace=ws), ref.product(q, sx, dense, sw, None, "fp16"))


@pytest.mark.parametrize("T", [1, 16, 80, 600])
def test_product_on_streams_and_in_a_graph(T):
    """Two streams at once, and a captured call replayed with other inputs between eager calls."""
    c, q, sx, sw, bias, dense, Q, SX = make(512, 1024, 64, 5, T, 21)
    want = ref.product(q, sx, dense, sw, None, "fp16")
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for k in range(6):
        with torch.cuda.stream(streams[k % 2]):
            got.append(vnm.vnm_spmm_i8(Q, SX, c))
    torch.cuda.synchronize()
    assert all(same(g, want) for g in got)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            graphs.append((g, vnm.vnm_spmm_i8(Q, SX, c)))
    rng = np.random.default_rng(5)
    for k in range(4):
        q2 = rng.integers(-128, 128, q.shape).astype(np.int8)
        Q.copy_(torch.from_numpy(q2).to(DEV))
        want = ref.product(q2, sx, dense, sw, None, "fp16")
        for g, y in graphs:
            g.replay()
        eager = vnm.vnm_spmm_i8(Q, SX, c)
        torch.cuda.synchronize()
        assert same(eager, want) and all(same(y, want) for _, y in graphs)


def test_scratch_memory_elsewhere_is_refused():
    """Memory on the host, with gaps, or of another type never reaches a kernel, however large it is."""
    c, _, _, _, _, _, Q, SX = make(256, 512, 64, 8, 700, 11)
    need = 1 << 24
    w = torch.ones(512, dtype=torch.float16, device=DEV)
    for bad in (torch.empty(need, dtype=torch.uint8), torch.empty(1, dtype=torch.uint8, device=DEV).expand(need),
                torch.empty(need // 4, dtype=torch.float32, device=DEV)):
        with pytest.raises(AssertionError):
            vnm.vnm_spmm_i8(Q, SX, c, workspace=bad)
        with pytest.raises(AssertionError):
            vnm.vnm_stage_q(Q, 8, staged=bad)
        with pytest.raises(AssertionError):
            vnm.vnm_spmm_i8_staged(bad, SX, c)
        with pytest.raises(AssertionError):
            vnm.vnm_residual_norm_backward(Q.half(), torch.zeros(700, 4, device=DEV), dx=Q.half(), pre="rms", pre_weight=w, workspace=bad)


# --- together ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("T", [1, 37, 200])
def test_block_of_int8_layers(T):
    """Norm and quantization, two pruned and quantized layers, and the norms behind them, as a block runs them."""
    n, f = 512, 1376
    W1, X = syn.make_weight_and_input(f, n, T, seed=1)
    W2, _ = syn.make_weight_and_input(n, f, 1, seed=2)
    layers = [vnm.vnm_quantize_compressed(vnm.vnm_prune_compress(torch.from_numpy(W).to(DEV), 64, 5)) for W in (W1, W2)]
    h = torch.from_numpy(X.astype(np.float32)).to(DEV)
    g = torch.Generator().manual_seed(3)
    w1, w2, gate = (torch.randn(n, generator=g).half().to(DEV) for _ in range(3))
    a = vnm.vnm_residual_norm(h, pre="rms", pre_weight=w1, x_dtype=torch.float16, int8=True)
    u = vnm.vnm_spmm_i8(a.x, a.scale, layers[0])
    q, s = vnm.vnm_quantize_x(torch.nn.functional.silu(u))
    y = vnm.vnm_spmm_i8(q, s, layers[1])
    b = vnm.vnm_residual_norm(a.h, y, gate=gate, post="layer", pre="rms", pre_weight=w2)
    # each step against its plain form on the inputs it was given
    h64, w64 = h.double().cpu(), [w.double().cpu() for w in (w1, w2, gate)]
    _, x64, _, _, mag = ref.residual_norm(h64, None, None, 1.0, ("none", None, None, 1e-5), ("rms", w64[0], None, 1e-5))
    assert torch.equal(a.h, h)
    # the scale is the largest of a token's values over 127; a value is within half a step of its own, plus fp32 errors
    # (192 of 2^-24 of the terms behind it: see the test of the norms)
    step = x64.abs().amax(1, keepdim=True) / 127
    assert bool(((a.x.cpu().double() * a.scale.cpu().double()[:, None] - x64).abs() <= step * (0.5 + 1e-5) + 192 * 2.0 ** -24 * mag).all())
    for layer, qq, ss, yy in ((layers[0], a.x, a.scale, u), (layers[1], q, s, y)):
        dense = np.zeros((layer.out, layer.inn))
        W = vnm.vnm_decompress(vnm.Compressed(layer.values.half(), layer.meta, layer.colidx, None, layer.out, layer.inn, 64, 5))
        dense = W.cpu().numpy().astype(np.int64)
        assert same(yy, ref.product(qq.cpu().numpy(), ss.cpu().numpy(), dense, layer.scale.cpu().numpy(), None, "fp16"))
    want_q, want_s = ref.quantize_rows(torch.nn.functional.silu(u).float().cpu().numpy())
    assert np.array_equal(q.cpu().numpy(), want_q) and same(s, torch.from_numpy(want_s))
    h2, x2, _, mh, mx = ref.residual_norm(h64, y.double().cpu(), w64[2], 1.0, ("layer", None, None, 1e-5), ("rms", w64[1], None, 1e-5))
    assert bool(((b.h.cpu().double() - h2).abs() <= 64 * 2.0 ** -24 * mh).all())
    # (2^-25: half of fp16's smallest step, 2^-24, which is what values below 2^-14 are rounded by)
    assert bool(((b.x.cpu().double() - x2).abs() <= 2.0 ** -11 * x2.abs() + 192 * 2.0 ** -24 * mx + 2.0 ** -25).all())


def test_int8_layer_is_near_the_fp16_layer():
    """Quantization moves a result by at most half a step per factor: |dy| <= sum |w| sx / 2 + |x| sw / 2 + sx sw / 4 over the kept weights."""
    W, X = syn.make_weight_and_input(256, 640, 50, seed=8)
    c = vnm.vnm_prune_compress(torch.from_numpy(W).to(DEV), 64, 5, want_mask=True)
    x = torch.from_numpy(X).to(DEV)
    y16 = vnm.vnm_spmm(x, c, out_dtype=torch.float32).cpu().double()
    q = vnm.vnm_quantize_compressed(c)
    a, s = vnm.vnm_quantize_x(x)
    y8 = vnm.vnm_spmm_i8(a, s, q, out_dtype=torch.float32).cpu().double()
    Wm, sw, sx = torch.from_numpy(orc.masked_dense(W, c.mask.cpu().numpy()).astype(np.float64)), q.scale.cpu().double(), s.cpu().double()
    mask, x64 = c.mask.cpu().double(), torch.from_numpy(X.astype(np.float64))
    bound = sx[:, None] / 2 * Wm.abs().sum(1)[None] + (x64.abs() @ mask.t()) * sw[None] / 2 + sx[:, None] * sw[None] / 4 * mask.sum(1)[None]
    # (and fp32 sums of the fp16 layer: 2^-24 for each of at most 640 terms)
    bound = bound * (1 + 1e-5) + 640 * 2.0 ** -24 * (x64.abs() @ Wm.abs().t())
    assert bool(((y8 - y16).abs() <= bound).all())
