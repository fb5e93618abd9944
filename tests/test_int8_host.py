"""The 8-bit layer and the norms on the host: refusals before anything touches a device, sizes, and the plain forms the GPU
tests compare with.  No GPU needed: pointers that are not null are never dereferenced by a call that is refused."""

import ctypes

import numpy as np
import pytest
import torch

import paper_2410_16135_amd as vnm
from paper_2410_16135_amd import binding
from tests import int8_reference as ref

P = ctypes.c_void_p
G = P(0x10000)                                       # a well-aligned address that nothing reads
OK, NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE = range(6)


@pytest.fixture(scope="module")
def lib():
    return vnm.load_library()


def test_quantize_refusals(lib):
    q = lib.vnm_quantize_x
    assert q(None, 0, 64, 64, 0, None, 64, None, None) == OK                         # no tokens, no tensors
    assert q(None, 4, 64, 64, 0, G, 64, G, None) == NULL
    assert q(G, 4, 64, 64, 0, None, 64, G, None) == NULL and q(G, 4, 64, 64, 0, G, 64, None, None) == NULL
    assert q(G, -1, 64, 64, 0, G, 64, G, None) == SHAPE and q(G, 4, 0, 64, 0, G, 64, G, None) == SHAPE
    assert q(G, 4, 64, 63, 0, G, 64, G, None) == SHAPE and q(G, 4, 64, 64, 0, G, 63, G, None) == SHAPE
    assert q(G, 4, 64, 64, 3, G, 64, G, None) == UNSUPPORTED and q(G, 4, 64, 64, -1, G, 64, G, None) == UNSUPPORTED
    assert q(P(0x10001), 4, 64, 64, 0, G, 64, G, None) == ALIGN and q(P(0x10002), 4, 64, 64, 1, G, 64, G, None) == ALIGN
    assert q(G, 4, 64, 64, 0, G, 64, P(0x10002), None) == ALIGN


def _product_args(**over):
    a = dict(Q=G, T=4, ldq=128, sx=G, values=G, meta=G, colidx=G, packed=G, sw=G, out=128, inn=128, V=64, N=2, M=8, bias=None,
             Y=G, ldy=128, y_dtype=0, path=0, ws=G, ws_bytes=1 << 30, stream=None)
    a.update(over)
    return list(a.values())


@pytest.mark.parametrize("over,status", [
    (dict(values=None), NULL), (dict(meta=None), NULL), (dict(colidx=None), NULL), (dict(sw=None), NULL), (dict(Q=None), NULL),
    (dict(sx=None), NULL), (dict(Y=None), NULL), (dict(T=-1), SHAPE), (dict(ldq=127), SHAPE), (dict(ldy=127), SHAPE),
    (dict(out=0), SHAPE), (dict(inn=-5), SHAPE), (dict(V=48), UNSUPPORTED), (dict(N=1), UNSUPPORTED), (dict(M=3), UNSUPPORTED),
    (dict(y_dtype=3), UNSUPPORTED), (dict(path=3), UNSUPPORTED), (dict(ws_bytes=-1), WORKSPACE), (dict(Y=P(0x10001)), ALIGN),
    (dict(Y=P(0x10002), y_dtype=1), ALIGN), (dict(sx=P(0x10002)), ALIGN), (dict(sw=P(0x10001)), ALIGN), (dict(bias=P(0x10001)), ALIGN),
    (dict(packed=P(0x10080)), ALIGN), (dict(path=2, packed=None), UNSUPPORTED), (dict(path=2, V=16), UNSUPPORTED),
    (dict(path=2, M=17), UNSUPPORTED), (dict(path=2, ldq=136), UNSUPPORTED), (dict(path=2, Q=P(0x10008)), UNSUPPORTED),
    # sums that could leave 32 bits: 2 * 65536 products of up to 2^14
    (dict(inn=65536 * 8, ldq=65536 * 8), UNSUPPORTED),
    (dict(T=0, Q=None, sx=None, Y=None), OK), (dict(T=0, Q=None, sx=None, Y=None, ws=None, ws_bytes=0), OK),
])
def test_product_refusals(lib, over, status):
    assert lib.vnm_spmm_i8(*_product_args(**over)) == status


def test_pack_and_sizes(lib):
    b = ctypes.c_int64(-1)
    assert lib.vnm_i8_packed_bytes(128, 128, 64, 2, 8, None) == NULL and lib.vnm_i8_packed_bytes(0, 128, 64, 2, 8, ctypes.byref(b)) == SHAPE
    for out, inn, V, M, has in ((128, 128, 64, 8, True), (100, 37, 32, 5, True), (128, 128, 16, 8, False), (128, 128, 64, 17, False)):
        assert lib.vnm_i8_packed_bytes(out, inn, V, 2, M, ctypes.byref(b)) == OK and (b.value > 0) == has
        # int8 values and positions of 64-row blocks at least
        assert not has or b.value >= -(-out // 64) * -(-inn // (16 * M)) * 2560
    assert lib.vnm_pack_i8(None, G, G, 128, 128, 64, 2, 8, G, None) == NULL and lib.vnm_pack_i8(G, G, G, 128, 128, 64, 2, 8, None, None) == NULL
    assert lib.vnm_pack_i8(G, G, G, 128, 128, 16, 2, 8, G, None) == UNSUPPORTED
    assert lib.vnm_pack_i8(G, G, G, 128, 128, 64, 2, 8, P(0x10010), None) == ALIGN
    qc = lib.vnm_quantize_compressed
    assert qc(None, G, G, 128, 128, 64, 2, 8, G, G, None, None) == NULL and qc(G, G, G, 128, 128, 64, 2, 8, G, None, None, None) == NULL
    assert qc(P(0x10001), G, G, 128, 128, 64, 2, 8, G, G, None, None) == ALIGN and qc(G, G, G, 128, 128, 64, 2, 8, G, P(0x10002), None, None) == ALIGN
    assert qc(G, G, G, 128, 128, 16, 2, 8, G, G, G, None) == UNSUPPORTED
    assert lib.vnm_spmm_i8_workspace_bytes(-1, 128, 128, 64, 2, 8, ctypes.byref(b)) == SHAPE
    assert lib.vnm_spmm_i8_workspace_bytes(4, 128, 128, 64, 2, 8, None) == NULL
    assert lib.vnm_spmm_i8_workspace_bytes(0, 128, 128, 64, 2, 8, ctypes.byref(b)) == OK and b.value >= 0


def test_staging_refusals(lib):
    b = ctypes.c_int64(-1)
    q = lib.vnm_stage_q_bytes
    assert q(4, 128, 8, None) == NULL and q(-1, 128, 8, ctypes.byref(b)) == SHAPE and q(4, 0, 8, ctypes.byref(b)) == SHAPE
    assert q(4, 128, 3, ctypes.byref(b)) == UNSUPPORTED and q(4, 128, 17, ctypes.byref(b)) == UNSUPPORTED
    # a tile of 128 tokens and the look-ahead: 16 M rows of 144 bytes, whole KiB, per step of 16 M columns
    assert q(4, 128, 8, ctypes.byref(b)) == OK and b.value == (1 + 5) * 18 * 1024
    need, st = b.value, lib.vnm_stage_q
    assert st(None, 0, 128, 128, 8, None, 0, None) == OK
    assert st(None, 4, 128, 128, 8, G, need, None) == NULL and st(G, 4, 128, 128, 8, None, need, None) == NULL
    assert st(G, 4, 127, 128, 8, G, need, None) == SHAPE and st(G, 4, 136, 128, 8, G, need, None) == UNSUPPORTED
    assert st(P(0x10008), 4, 128, 128, 8, G, need, None) == UNSUPPORTED and st(G, 4, 128, 128, 17, G, need, None) == UNSUPPORTED
    assert st(G, 4, 128, 128, 8, G, need - 1, None) == WORKSPACE and st(G, 4, 128, 128, 8, P(0x10080), need, None) == ALIGN

    def product(**over):
        a = dict(staged=G, bytes=need, T=4, sx=G, packed=G, sw=G, out=128, inn=128, V=64, N=2, M=8, bias=None, Y=G, ldy=128, y_dtype=0, stream=None)
        a.update(over)
        return lib.vnm_spmm_i8_staged(*a.values())

    assert product(T=0, staged=None, bytes=0, sx=None, Y=None) == OK
    for name in ("staged", "sx", "packed", "sw", "Y"):
        assert product(**{name: None}) == NULL, name
    assert product(T=-1) == SHAPE and product(ldy=127) == SHAPE and product(out=0) == SHAPE
    assert product(y_dtype=4) == UNSUPPORTED and product(V=16) == UNSUPPORTED and product(M=17) == UNSUPPORTED
    assert product(inn=65536 * 8, bytes=1 << 60) == UNSUPPORTED and product(bytes=need - 1) == WORKSPACE
    for name, at in (("staged", 0x10010), ("packed", 0x10080), ("sx", 0x10002), ("sw", 0x10002), ("bias", 0x10001), ("Y", 0x10001)):
        assert product(**{name: P(at)}) == ALIGN, name


def _forward_args(**over):
    f = dict(T=4, n=64, h_dtype=0, x_dtype=0, post=0, pre=1, post_eps=1e-5, pre_eps=1e-5, residual_scale=1.0, gate_tokens=0, h=0x10000,
             ldh=64, ldy=64, ldg=64, h_out=0x20000, x=0x30000, ldho=64, ldx=64, ldq=64)
    f.update(over)
    return binding._ResidualNormArgs(**f)


@pytest.mark.parametrize("over,status", [
    (dict(h=None), NULL), (dict(h_out=None, x=None), NULL), (dict(x=None, q=0x30000), NULL), (dict(q=0x40000, q_scale=0x50000), UNSUPPORTED),
    (dict(gate=0x60000), NULL), (dict(post=1), NULL), (dict(T=-1), SHAPE), (dict(n=0), SHAPE), (dict(gate_tokens=-1), SHAPE),
    (dict(ldh=63), SHAPE), (dict(ldho=63), SHAPE), (dict(ldx=63), SHAPE), (dict(y=0x60000, ldy=63), SHAPE),
    (dict(y=0x60000, gate=0x70000, gate_tokens=2, ldg=63), SHAPE), (dict(h_out=0x10000, ldho=72), SHAPE),
    (dict(n=16385, ldh=20000, ldho=20000, ldx=20000), UNSUPPORTED), (dict(x_dtype=2), UNSUPPORTED), (dict(h_dtype=3), UNSUPPORTED),
    (dict(h_dtype=0, x_dtype=1), UNSUPPORTED), (dict(pre=3), UNSUPPORTED), (dict(post=-1), UNSUPPORTED), (dict(pre_eps=0.0), UNSUPPORTED),
    (dict(pre_eps=float("nan")), UNSUPPORTED), (dict(y=0x60000, post=2, post_eps=-1.0), UNSUPPORTED), (dict(pre=0, pre_weight=0x60000), UNSUPPORTED),
    (dict(post_bias=0x60000), UNSUPPORTED), (dict(h=0x10001), ALIGN), (dict(h_dtype=1, h=0x10002), ALIGN), (dict(x=0x30001), ALIGN),
    (dict(pre_weight=0x60001), ALIGN), (dict(stats=0x60008), ALIGN), (dict(x=None, q=0x40000, q_scale=0x50001), ALIGN),
    (dict(T=0, h=None, x=None, h_out=None), OK),
])
def test_norm_refusals(lib, over, status):
    assert lib.vnm_residual_norm(ctypes.byref(_forward_args(**over)), None) == status


def _backward_args(**over):
    f = dict(T=4, n=64, h_dtype=0, x_dtype=0, post=0, pre=1, residual_scale=1.0, gate_tokens=0, dx=0x10000, dh_out=0x20000, h_new=0x30000,
             stats=0x40000, lddx=64, lddho=64, ldh=64, ldy=64, ldg=64, dh=0x50000, lddh=64, lddy=64)
    f.update(over)
    return binding._ResidualNormBackwardArgs(**f)


@pytest.mark.parametrize("over,status", [
    (dict(dx=None, dh_out=None), NULL), (dict(dh=None), NULL), (dict(h_new=None), NULL), (dict(stats=None), NULL),
    (dict(dy=0x60000, post=1), NULL), (dict(d_gate=0x60000), NULL), (dict(T=-1), SHAPE), (dict(n=0), SHAPE), (dict(lddx=63), SHAPE),
    (dict(lddho=63), SHAPE), (dict(ldh=63), SHAPE), (dict(lddh=63), SHAPE), (dict(dy=0x60000, lddy=63), SHAPE),
    (dict(dh=0x20000, lddh=72), SHAPE), (dict(n=16385, lddx=20000, lddho=20000, ldh=20000, lddh=20000), UNSUPPORTED),
    (dict(x_dtype=2), UNSUPPORTED), (dict(d_post_weight=0x60000), UNSUPPORTED), (dict(pre=0, d_pre_weight=0x60000), UNSUPPORTED),
    (dict(post=7), UNSUPPORTED), (dict(dx=0x10001), ALIGN), (dict(d_pre_weight=0x60002), ALIGN), (dict(stats=0x40004), ALIGN),
    (dict(d_pre_weight=0x60000), WORKSPACE),
])
def test_norm_backward_refusals(lib, over, status):
    assert lib.vnm_residual_norm_backward(ctypes.byref(_backward_args(**over)), None, 0, None) == status


def test_norm_backward_workspace(lib):
    b = ctypes.c_int64(0)
    w = lib.vnm_residual_norm_backward_workspace_bytes
    assert w(16, 64, 0, None) == NULL and w(-1, 64, 0, ctypes.byref(b)) == SHAPE and w(16, 0, 0, ctypes.byref(b)) == SHAPE
    assert w(16, 16385, 0, ctypes.byref(b)) == UNSUPPORTED
    assert w(16, 64, 0, ctypes.byref(b)) == OK and b.value > 0
    args = ctypes.byref(_backward_args(d_pre_weight=0x60000))
    assert lib.vnm_residual_norm_backward(args, G, 16, None) == WORKSPACE and lib.vnm_residual_norm_backward(args, G, -1, None) == WORKSPACE
    assert lib.vnm_residual_norm_backward(args, P(0x10004), b.value, None) == ALIGN


def test_binding_refuses_other_types():
    with pytest.raises(vnm.VnmError):
        binding._dtype_code(torch.float64)
    with pytest.raises(AssertionError):
        vnm.vnm_quantize_x(torch.zeros(4, 8))                 # not on a GPU
    with pytest.raises(AssertionError):
        vnm.vnm_residual_norm(torch.zeros(4, 8))


def test_plain_quantization():
    q, s = ref.quantize_rows(np.array([[1, -127, 63.5, 0.5], [0, 0, 0, 0], [1, np.inf, 0, 0], [np.nan, 1, 2, 3]], np.float32))
    assert q.tolist() == [[1, -127, 64, 0], [0] * 4, [0] * 4, [0] * 4]        # halves go to the even neighbour
    assert s[0] == 1 and s[1] == 0 and np.isnan(s[2:]).all()


def test_plain_product_takes_the_kept_columns():
    rng = np.random.default_rng(0)
    values, meta, col, scale, dense = ref.random_triple(rng, 20, 23, 16, 6)
    for o in (0, 15, 16, 19):
        for b in range(4):
            byte = int(meta[o, b // 2])
            nib = byte >> 4 if b % 2 else byte & 15
            want = np.zeros(6, np.int64)
            want[col[o // 16, b, nib & 3]], want[col[o // 16, b, nib >> 2]] = values[o, b]
            assert (dense[o, 6 * b:6 * b + 6] == want[:len(dense[o, 6 * b:6 * b + 6])]).all()


def test_plain_norm_agrees_with_torch():
    g = torch.Generator().manual_seed(0)
    v, w, b = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((5, 33), (33,), (33,)))
    got = ref.normed(v, "layer", w, b, 1e-5)[0]
    assert torch.allclose(got, torch.nn.functional.layer_norm(v, (33,), w, b, 1e-5), rtol=1e-12, atol=1e-12)
