"""ctypes binding of include/vnm.h.  PyTorch is used for device memory and streams only."""

from __future__ import annotations

import ctypes
import functools
import os
import struct
from dataclasses import dataclass
from typing import NamedTuple

PATH_AUTO, PATH_GENERIC, PATH_SMFMAC = 0, 1, 2

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
_LIB = None


class VnmError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(what)


class VnmSizes(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in (
        "out_pad", "in_pad", "row_blocks", "col_blocks", "kc", "values_elems", "meta_bytes",
        "colidx_bytes", "packed_bytes", "workspace_bytes")]


def _struct(name, *groups):
    """A ctypes structure from (type, "field field ...") pairs."""
    return type(name, (ctypes.Structure,), {"_fields_": [(f, t) for t, names in groups for f in names.split()]})


_I64, _INT, _F32, _PTR = ctypes.c_int64, ctypes.c_int, ctypes.c_float, ctypes.c_void_p
_ResidualNormArgs = _struct(
    "_ResidualNormArgs", (_I64, "T n"), (_INT, "h_dtype x_dtype post pre"), (_F32, "post_eps pre_eps residual_scale"),
    (_I64, "gate_tokens"), (_PTR, "h y gate post_weight post_bias pre_weight pre_bias"), (_I64, "ldh ldy ldg"),
    (_PTR, "h_out x q q_scale stats"), (_I64, "ldho ldx ldq"))
_ResidualNormBackwardArgs = _struct(
    "_ResidualNormBackwardArgs", (_I64, "T n"), (_INT, "h_dtype x_dtype post pre"), (_F32, "residual_scale"),
    (_I64, "gate_tokens"), (_PTR, "dx dh_out h_new y gate post_weight post_bias pre_weight stats"),
    (_I64, "lddx lddho ldh ldy ldg"), (_PTR, "dh dy d_post_weight d_post_bias d_pre_weight d_pre_bias d_gate"),
    (_I64, "lddh lddy"))


# The same bytes from struct.pack, which a call on few tokens builds in a third of the time
_NORM_ARGS = struct.Struct("@2q4i3f4xq" + "7P3q" + "5P3q")
_NORM_BACKWARD_ARGS = struct.Struct("@2q4if4xq" + "9P5q" + "7P2q")
assert _NORM_ARGS.size == ctypes.sizeof(_ResidualNormArgs) and _NORM_BACKWARD_ARGS.size == ctypes.sizeof(_ResidualNormBackwardArgs)


def lib_path() -> str:
    """The in-tree library."""
    return os.path.join(_PKG_DIR, "libvnm.so")


def load_library():
    """Load libvnm.so.  The library carries a hash of the sources it was built from; when it is
    missing, or the sources have changed since, it is rebuilt first (hipcc needed), so results never
    come from kernels that are no longer in the tree.  Raises if neither works."""
    global _LIB
    if _LIB is not None:
        return _LIB
    from .build import build_library, built_hash, source_hash
    path = lib_path()
    want = source_hash()
    if built_hash(path) != want:
        import sys
        print("libvnm.so is missing or older than its sources: rebuilding", file=sys.stderr, flush=True)
        build_library()
        if built_hash(path) != want:
            raise VnmError(-1, "libvnm.so does not match its sources even after a rebuild")
    lib = ctypes.CDLL(path)
    lib.vnm_source_hash.restype = ctypes.c_char_p
    if lib.vnm_source_hash().decode() != want:
        raise VnmError(-1, "the loaded libvnm.so reports a different source hash than its file")
    vp, i64, ci = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
    lib.vnm_query_sizes.argtypes = [i64, i64, ci, ci, ci, ctypes.POINTER(VnmSizes)]
    lib.vnm_prune_compress.argtypes = [vp, i64, i64, i64, ci, ci, ci, vp, vp, vp, vp, vp, vp, i64, vp]
    lib.vnm_pack.argtypes = [vp, vp, vp, i64, i64, ci, ci, ci, vp, vp]
    lib.vnm_spmm.argtypes = [vp, i64, i64, vp, vp, vp, vp, i64, i64, ci, ci, ci, vp, i64, ci, ci, vp, i64, vp]
    lib.vnm_spmm_noalloc.argtypes = [vp, i64, i64, vp, vp, vp, vp, i64, i64, ci, ci, ci, vp, i64, ci, ci, vp]
    lib.vnm_spmm_noalloc.restype = ci
    lib.vnm_spmm_fused.argtypes = [vp, i64, i64, vp, vp, vp, vp, i64, i64, ci, ci, ci, vp, vp, vp, vp, i64, ci, ci,
                                   vp, i64, vp]
    lib.vnm_spmm_fused.restype = ci
    lib.vnm_spmm_fused_workspace_bytes.argtypes = [i64, i64, i64, ci, ci, ci, ci, ctypes.POINTER(i64)]
    lib.vnm_spmm_fused_workspace_bytes.restype = ci
    cd = ctypes.c_double
    lib.vnm_permutation_search_workspace_bytes.argtypes = [i64, i64, ci, ci, ci, ctypes.POINTER(i64)]
    lib.vnm_permutation_search_workspace_bytes.restype = ci
    lib.vnm_permutation_search.argtypes = [vp, i64, i64, i64, ci, ci, ci, cd, ci, vp, vp, vp, vp, i64, vp]
    lib.vnm_permutation_search.restype = ci
    lib.vnm_permutation_gain.argtypes = [vp, i64, i64, i64, ci, ci, ci, cd, ci, ci, vp, vp, vp, vp, i64, vp]
    lib.vnm_permutation_gain.restype = ci
    lib.vnm_retained_score.argtypes = [vp, i64, i64, i64, ci, ci, ci, cd, vp, vp, ctypes.POINTER(i64), vp, i64, vp]
    lib.vnm_retained_score.restype = ci
    lib.vnm_lora_merge.argtypes = [vp, i64, i64, i64, vp, i64, vp, i64, ci, ctypes.c_float, vp, i64, vp]
    lib.vnm_lora_merge.restype = ci
    lib.vnm_refresh_mask_workspace_bytes.argtypes = [i64, i64, ci, ci, ci, ctypes.POINTER(i64)]
    lib.vnm_refresh_mask_workspace_bytes.restype = ci
    lib.vnm_refresh_mask.argtypes = [vp, i64, i64, i64, vp, i64, vp, i64, ci, ctypes.c_float, vp, ci, ci, ci, vp, i64, vp,
                                     vp, vp, vp, vp, vp, i64, vp]
    lib.vnm_refresh_mask.restype = ci
    lib.vnm_lsa_max.argtypes = [vp, ci, vp, ctypes.POINTER(i64)]
    lib.vnm_lsa_max.restype = ci
    lib.vnm_lsa_max_method.argtypes = [vp, ci, ci, vp, ctypes.POINTER(i64)]
    lib.vnm_lsa_max_method.restype = ci
    lib.vnm_fold_permutations.argtypes = [vp, vp, i64, vp]
    lib.vnm_fold_permutations.restype = ci
    lib.vnm_decompress.argtypes = [vp, vp, vp, i64, i64, ci, ci, ci, vp, i64, vp]
    lib.vnm_stage_x.argtypes = [vp, i64, i64, i64, ci, vp, i64, vp]
    lib.vnm_spmm_staged.argtypes = [vp, i64, i64, vp, i64, i64, ci, ci, ci, vp, i64, ci, vp, i64, vp]
    lib.vnm_stage_x.restype = ci
    lib.vnm_spmm_staged.restype = ci
    lib.vnm_spmm_kernel_choice.argtypes = [i64, i64, i64, ci, ci, ci, i64, ctypes.POINTER(ci)]
    lib.vnm_spmm_kernel_choice.restype = ci
    lib.vnm_spmm_workspace_bytes.argtypes = [i64, i64, i64, ci, ci, ci, ctypes.POINTER(i64)]
    lib.vnm_spmm_workspace_bytes.restype = ci
    lib.vnm_ria_scores.argtypes = [vp, i64, i64, i64, vp, vp, i64, vp, i64, vp]
    lib.vnm_ria_scores.restype = ci
    lib.vnm_prune_compress_scored.argtypes = [vp, vp, i64, i64, i64, i64, ci, ci, ci, vp, vp, vp, vp, vp, vp]
    lib.vnm_prune_compress_scored.restype = ci
    lib.vnm_mask_diversity_log.argtypes = [ci, ci, ci, ctypes.POINTER(ctypes.c_double)]
    lib.vnm_mask_diversity_log.restype = ci
    lib.vnm_select_vm.argtypes = [ctypes.POINTER(ci), ctypes.POINTER(ci), ctypes.POINTER(ctypes.c_double), ci,
                                  ctypes.c_double, ctypes.POINTER(ci)]
    lib.vnm_select_vm.restype = ci
    lib.vnm_stage_x_bytes.argtypes = [i64, i64, ci, ctypes.POINTER(i64)]
    lib.vnm_stage_x_bytes.restype = ci
    lib.vnm_spmm_scratch_bytes.argtypes = [i64, i64, ctypes.POINTER(i64)]
    lib.vnm_spmm_scratch_bytes.restype = ci
    for f in (lib.vnm_query_sizes, lib.vnm_prune_compress, lib.vnm_pack, lib.vnm_spmm, lib.vnm_decompress,
              lib.vnm_format_version):
        f.restype = ci
    lib.vnm_quantize_x.argtypes = [vp, i64, i64, i64, ci, vp, i64, vp, vp]
    lib.vnm_i8_packed_bytes.argtypes = [i64, i64, ci, ci, ci, ctypes.POINTER(i64)]
    lib.vnm_quantize_compressed.argtypes = [vp, vp, vp, i64, i64, ci, ci, ci, vp, vp, vp, vp]
    lib.vnm_pack_i8.argtypes = [vp, vp, vp, i64, i64, ci, ci, ci, vp, vp]
    lib.vnm_spmm_i8.argtypes = [vp, i64, i64, vp, vp, vp, vp, vp, vp, i64, i64, ci, ci, ci, vp, vp, i64, ci, ci, vp, i64, vp]
    lib.vnm_spmm_i8_workspace_bytes.argtypes = [i64, i64, i64, ci, ci, ci, ctypes.POINTER(i64)]
    lib.vnm_stage_q_bytes.argtypes = [i64, i64, ci, ctypes.POINTER(i64)]
    lib.vnm_stage_q.argtypes = [vp, i64, i64, i64, ci, vp, i64, vp]
    lib.vnm_spmm_i8_staged.argtypes = [vp, i64, i64, vp, vp, vp, i64, i64, ci, ci, ci, vp, vp, i64, ci, vp]
    lib.vnm_residual_norm.argtypes = [vp, vp]
    lib.vnm_residual_norm_backward.argtypes = [vp, vp, i64, vp]
    lib.vnm_residual_norm_backward_workspace_bytes.argtypes = [i64, i64, i64, ctypes.POINTER(i64)]
    for f in (lib.vnm_quantize_x, lib.vnm_i8_packed_bytes, lib.vnm_quantize_compressed, lib.vnm_pack_i8, lib.vnm_spmm_i8,
              lib.vnm_spmm_i8_workspace_bytes, lib.vnm_stage_q_bytes, lib.vnm_stage_q, lib.vnm_spmm_i8_staged, lib.vnm_residual_norm, lib.vnm_residual_norm_backward,
              lib.vnm_residual_norm_backward_workspace_bytes):
        f.restype = ci
    lib.vnm_status_string.argtypes = [ci]
    lib.vnm_status_string.restype = ctypes.c_char_p
    lib.vnm_last_hip_error.restype = ctypes.c_char_p
    _LIB = lib
    return lib


def _check(status: int, what: str):
    if status != 0:
        lib = load_library()
        msg = lib.vnm_status_string(status).decode()
        detail = lib.vnm_last_hip_error().decode()
        if status == 6 or (status == 5 and what == "vnm_spmm_noalloc" and detail):
            msg += " (" + detail + ")"
        raise VnmError(status, f"{what}: {msg}")


# A call on a small layer is bound by what happens here, not by its kernel (128 x 128 at 16 tokens: 7 us on the device).
# Addresses and streams are therefore passed as plain integers, the stream is asked for without building a Stream object,
# and the size queries, functions of a few integers, are answered from a bounded cache: 11.7 -> 8.6 us per call there.
def _ptr(t):
    return 0 if t is None else t.data_ptr()


def _raw_stream(device) -> int:
    """The current stream of a CUDA device as an integer."""
    global _raw_stream
    import torch
    get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if get is None:
        def _raw_stream(device):
            return torch.cuda.current_stream(device).cuda_stream
    else:
        def _raw_stream(device):
            return get(device.index)
    return _raw_stream(device)


def _stream(t):
    return _raw_stream(t.device)


def vnm_query_sizes(out: int, inn: int, V: int, M: int, N: int = 2) -> VnmSizes:
    s = VnmSizes()
    _check(load_library().vnm_query_sizes(out, inn, V, N, M, ctypes.byref(s)), "vnm_query_sizes")
    return s


@dataclass
class Compressed:
    """The compressed triple of one layer plus the opaque matrix-core copy (device tensors)."""
    values: object
    meta: object
    colidx: object
    packed: object
    out: int
    inn: int
    V: int
    M: int
    mask: object = None


def _alloc(sizes: VnmSizes, device, want_packed=True):
    import torch
    values = torch.empty(sizes.values_elems, dtype=torch.float16, device=device)
    meta = torch.empty(sizes.meta_bytes, dtype=torch.uint8, device=device)
    colidx = torch.empty(sizes.colidx_bytes, dtype=torch.uint8, device=device)
    packed = None
    if want_packed and sizes.packed_bytes > 0:
        packed = torch.empty(sizes.packed_bytes, dtype=torch.uint8, device=device)
    return values, meta, colidx, packed


def vnm_prune_compress(W, V: int, M: int, N: int = 2, want_mask: bool = False, want_packed: bool = True,
                       out=None) -> Compressed:
    """W: fp16 CUDA tensor [out x in] (row stride may exceed `in`).  Allocates the outputs (or
    reuses `out`, a Compressed of the same layer) and enqueues the kernel on the current stream."""
    import torch
    assert W.is_cuda and W.dtype == torch.float16 and W.dim() == 2 and W.stride(1) == 1
    o, i = W.shape
    sizes = vnm_query_sizes(o, i, V, M, N)
    if out is None:
        values, meta, colidx, packed = _alloc(sizes, W.device, want_packed)
        mask = torch.empty((o, i), dtype=torch.uint8, device=W.device) if want_mask else None
        out = Compressed(values, meta, colidx, packed, o, i, V, M, mask)
    _check(load_library().vnm_prune_compress(
        _ptr(W), o, i, W.stride(0), V, N, M, _ptr(out.values), _ptr(out.meta), _ptr(out.colidx),
        _ptr(out.mask), _ptr(out.packed), None, 0, _stream(W)), "vnm_prune_compress")
    return out


def vnm_ria_scores(W, act, S=None):
    """fp32 RIA scores [out x in] of W (fp16 CUDA) for the activation factors act (fp32 CUDA [in])."""
    import torch
    assert W.is_cuda and W.dtype == torch.float16 and W.dim() == 2 and W.stride(1) == 1
    assert act.is_cuda and act.dtype == torch.float32 and act.shape == (W.shape[1],) and act.is_contiguous()
    o, i = W.shape
    if S is None:
        S = torch.empty((o, i), dtype=torch.float32, device=W.device)
    ws = torch.empty((o + i) * 8, dtype=torch.uint8, device=W.device)
    _check(load_library().vnm_ria_scores(_ptr(W), o, i, W.stride(0), _ptr(act), _ptr(S), S.stride(0), _ptr(ws),
                                         ws.numel(), _stream(W)), "vnm_ria_scores")
    return S


def vnm_prune_compress_scored(W, S, V: int, M: int, N: int = 2, want_mask: bool = False,
                              want_packed: bool = True, out=None) -> Compressed:
    """vnm_prune_compress driven by the fp32 score matrix S [out x in] instead of |W|."""
    import torch
    assert W.is_cuda and W.dtype == torch.float16 and W.dim() == 2 and W.stride(1) == 1
    assert S.is_cuda and S.dtype == torch.float32 and S.shape == W.shape and S.stride(1) == 1
    o, i = W.shape
    sizes = vnm_query_sizes(o, i, V, M, N)
    if out is None:
        values, meta, colidx, packed = _alloc(sizes, W.device, want_packed)
        mask = torch.empty((o, i), dtype=torch.uint8, device=W.device) if want_mask else None
        out = Compressed(values, meta, colidx, packed, o, i, V, M, mask)
    _check(load_library().vnm_prune_compress_scored(
        _ptr(W), _ptr(S), o, i, W.stride(0), S.stride(0), V, N, M, _ptr(out.values), _ptr(out.meta),
        _ptr(out.colidx), _ptr(out.mask), _ptr(out.packed), _stream(W)), "vnm_prune_compress_scored")
    return out


def vnm_pack(c: Compressed, N: int = 2) -> Compressed:
    import torch
    sizes = vnm_query_sizes(c.out, c.inn, c.V, c.M, N)
    if c.packed is None:
        c.packed = torch.empty(sizes.packed_bytes, dtype=torch.uint8, device=c.values.device)
    _check(load_library().vnm_pack(_ptr(c.values), _ptr(c.meta), _ptr(c.colidx), c.out, c.inn, c.V, N, c.M,
                                   _ptr(c.packed), _stream(c.values)), "vnm_pack")
    return c


@functools.lru_cache(maxsize=1024, typed=True)      # (typed: 16.0 is refused, also after 16)
def _spmm_workspace_bytes(T: int, out: int, inn: int, V: int, N: int, M: int) -> int:
    b = ctypes.c_int64(0)
    _check(load_library().vnm_spmm_workspace_bytes(T, out, inn, V, N, M, ctypes.byref(b)), "vnm_spmm_workspace_bytes")
    return b.value


@functools.lru_cache(maxsize=1024, typed=True)      # (typed: 16.0 is refused, also after 16)
def _spmm_fused_workspace_bytes(T: int, out: int, inn: int, V: int, N: int, M: int, with_perm_in: int) -> int:
    b = ctypes.c_int64(0)
    _check(load_library().vnm_spmm_fused_workspace_bytes(T, out, inn, V, N, M, with_perm_in, ctypes.byref(b)),
           "vnm_spmm_fused_workspace_bytes")
    return b.value


def vnm_spmm_workspace_bytes(T: int, c: Compressed, N: int = 2) -> int:
    return _spmm_workspace_bytes(T, c.out, c.inn, c.V, N, c.M)


_WORKSPACES = {}


def _workspace(device, nbytes: int):
    """One grow-only scratch tensor per device, shared by all vnm_spmm calls of this process.
    Its reuse is ordered by the stream the calls run on: callers that use several streams at once
    must hand every call a `workspace` of its own."""
    import torch
    ws = _WORKSPACES.get(device)
    if ws is None or ws.numel() < nbytes:
        dev = device[0] if isinstance(device, tuple) else device
        ws = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=dev)
        _WORKSPACES[device] = ws
    return ws


def vnm_spmm(X, c: Compressed, N: int = 2, out_dtype=None, path: int = PATH_AUTO, Y=None, workspace=None):
    """Y [T x out] = X [T x in] . W'^T on the compressed weight; fp16 in, fp32 accumulate.
    `workspace`: optional uint8 CUDA tensor of at least vnm_spmm_workspace_bytes(T, c) bytes;
    by default a process-wide grow-only scratch tensor is used."""
    import torch
    assert X.is_cuda and X.dtype == torch.float16 and X.dim() == 2 and X.stride(1) == 1
    T = X.shape[0]
    assert X.shape[1] == c.inn
    if Y is None:
        Y = torch.empty((T, c.out), dtype=out_dtype or torch.float16, device=X.device)
    y_dtype = {torch.float16: 0, torch.float32: 1}[Y.dtype]
    ws, ws_bytes = None, 0
    if path != PATH_GENERIC and c.packed is not None and T > 0:
        ws_bytes = vnm_spmm_workspace_bytes(T, c, N)
        ws = workspace if workspace is not None else _workspace(X.device, ws_bytes)
        ws_bytes = ws.numel()
    _check(load_library().vnm_spmm(
        _ptr(X), T, X.stride(0) if T > 0 else c.inn, _ptr(c.values), _ptr(c.meta), _ptr(c.colidx),
        _ptr(c.packed), c.out, c.inn, c.V, N, c.M, _ptr(Y), Y.stride(0) if T > 0 else c.out, y_dtype, path,
        _ptr(ws), ws_bytes, _stream(X)), "vnm_spmm")
    return Y


def vnm_spmm_bind(X, c: Compressed, Y, workspace, N: int = 2, path: int = PATH_AUTO):
    """The vnm_spmm call on these buffers with its arguments marshalled once: returns a function of
    no arguments that issues the call on torch's current stream (a loop that serves the same layer
    again and again -- decoding -- pays the argument conversion once, not per call).  The tensors
    must stay alive and in place while the function is used."""
    import torch
    assert X.is_cuda and X.dtype == torch.float16 and X.dim() == 2 and X.stride(1) == 1
    T = X.shape[0]
    assert T > 0 and X.shape[1] == c.inn and Y.shape == (T, c.out) and Y.stride(1) == 1
    y_dtype = {torch.float16: 0, torch.float32: 1}[Y.dtype]
    fn = load_library().vnm_spmm
    vp = lambda t: ctypes.c_void_p(_ptr(t))
    args = (vp(X), ctypes.c_int64(T), ctypes.c_int64(X.stride(0)), vp(c.values), vp(c.meta), vp(c.colidx),
            vp(c.packed), ctypes.c_int64(c.out), ctypes.c_int64(c.inn), ctypes.c_int(c.V), ctypes.c_int(N),
            ctypes.c_int(c.M), vp(Y), ctypes.c_int64(Y.stride(0)), ctypes.c_int(y_dtype), ctypes.c_int(path),
            vp(workspace), ctypes.c_int64(0 if workspace is None else workspace.numel()))
    dev = X.device
    keep = (X, c, Y, workspace)

    def call():
        rc = fn(*args, _raw_stream(dev))
        if rc:
            _check(rc, "vnm_spmm")
        return keep[2]
    return call


NOALLOC_SCRATCH_BYTES = 32 << 20


def vnm_spmm_noalloc(X, c: Compressed, Y, N: int = 2, path: int = PATH_AUTO):
    """vnm_spmm into a caller-supplied Y with the library's built-in scratch instead of a workspace:
    the call allocates nothing (for callers that cannot: graph capture, serving loops)."""
    import torch
    assert X.is_cuda and X.dtype == torch.float16 and X.dim() == 2 and X.stride(1) == 1
    T = X.shape[0]
    assert X.shape[1] == c.inn and Y.shape == (T, c.out) and Y.stride(1) == 1
    y_dtype = {torch.float16: 0, torch.float32: 1}[Y.dtype]
    _check(load_library().vnm_spmm_noalloc(
        _ptr(X), T, X.stride(0) if T > 0 else c.inn, _ptr(c.values), _ptr(c.meta), _ptr(c.colidx),
        _ptr(c.packed), c.out, c.inn, c.V, N, c.M, _ptr(Y), Y.stride(0) if T > 0 else c.out, y_dtype, path,
        _stream(X)), "vnm_spmm_noalloc")
    return Y


def vnm_spmm_fused(X, c: Compressed, bias=None, perm_in=None, perm_out=None, N: int = 2, out_dtype=None,
                   path: int = PATH_AUTO, Y=None, workspace=None):
    """vnm_spmm with an optional bias (fp16 [out], row order of the compressed weight) and the two
    channel permutations of Eq. 6 (int32 CUDA tensors): Y[t, perm_out[o]] = bias[o] + sum_i W'[o, i]
    X[t, perm_in[i]].  If perm_out is not a permutation, untouched columns of a fresh Y are undefined."""
    import torch
    assert X.is_cuda and X.dtype == torch.float16 and X.dim() == 2 and X.stride(1) == 1
    T = X.shape[0]
    assert X.shape[1] == c.inn
    for name, p, n, dt in (("bias", bias, c.out, torch.float16), ("perm_in", perm_in, c.inn, torch.int32),
                           ("perm_out", perm_out, c.out, torch.int32)):
        assert p is None or (p.is_cuda and p.dtype == dt and p.is_contiguous() and p.numel() == n), name
    if Y is None:
        Y = torch.empty((T, c.out), dtype=out_dtype or torch.float16, device=X.device)
    y_dtype = {torch.float16: 0, torch.float32: 1}[Y.dtype]
    ws, ws_bytes = None, 0
    if path != PATH_GENERIC and c.packed is not None and T > 0:
        need = _spmm_fused_workspace_bytes(T, c.out, c.inn, c.V, N, c.M, int(perm_in is not None))
        ws = workspace if workspace is not None else _workspace(X.device, need)
        ws_bytes = ws.numel()
    _check(load_library().vnm_spmm_fused(
        _ptr(X), T, X.stride(0) if T > 0 else c.inn, _ptr(c.values), _ptr(c.meta), _ptr(c.colidx),
        _ptr(c.packed), c.out, c.inn, c.V, N, c.M, _ptr(bias), _ptr(perm_in), _ptr(perm_out), _ptr(Y),
        Y.stride(0) if T > 0 else c.out, y_dtype, path, _ptr(ws), ws_bytes, _stream(X)), "vnm_spmm_fused")
    return Y


def vnm_fold_permutations(perm_out_prev, perm_in_next):
    """Host: input permutation of the next layer when the previous one leaves its output in the
    row order of its (permuted) weight; int32 numpy arrays in, int32 numpy array out."""
    import numpy as np
    po = np.ascontiguousarray(perm_out_prev, dtype=np.int32)
    pi = np.ascontiguousarray(perm_in_next, dtype=np.int32)
    assert po.ndim == 1 and po.shape == pi.shape
    res = np.empty_like(po)
    _check(load_library().vnm_fold_permutations(po.ctypes.data, pi.ctypes.data, po.size, res.ctypes.data),
           "vnm_fold_permutations")
    return res


def _ps_workspace(S, V, M, N):
    import torch
    b = ctypes.c_int64(0)
    _check(load_library().vnm_permutation_search_workspace_bytes(S.shape[0], S.shape[1], V, N, M, ctypes.byref(b)),
           "vnm_permutation_search_workspace_bytes")
    return _workspace((S.device, "permsearch"), b.value)


def _host_perm(p, n):
    import numpy as np
    if p is None:
        return None, None
    a = np.ascontiguousarray(p, dtype=np.int32)
    assert a.shape == (n,)
    return a, a.ctypes.data


def vnm_permutation_search(S, V: int, M: int, scale: float, iterations: int = 2, N: int = 2):
    """Channel-permutation search of Eqs. 7-9 on the fp32 CUDA score matrix S.  Returns
    (perm_out, perm_in, history) as numpy arrays (int32, int32, int64)."""
    import numpy as np
    import torch
    assert S.is_cuda and S.dtype == torch.float32 and S.dim() == 2 and S.stride(1) == 1
    out, inn = S.shape
    ws = _ps_workspace(S, V, M, N)
    po, pi = np.empty(out, dtype=np.int32), np.empty(inn, dtype=np.int32)
    hist = np.zeros(1 + 2 * iterations, dtype=np.int64)
    _check(load_library().vnm_permutation_search(_ptr(S), out, inn, S.stride(0), V, N, M, float(scale), iterations,
                                                 po.ctypes.data, pi.ctypes.data, hist.ctypes.data, _ptr(ws),
                                                 ws.numel(), _stream(S)), "vnm_permutation_search")
    return po, pi, hist


def vnm_permutation_gain(S, V: int, M: int, scale: float, which: int, slot: int, perm_out=None, perm_in=None,
                         N: int = 2):
    """One gain matrix of the search (which: 0 input half-step, 1 output half-step); int64 numpy."""
    import numpy as np
    out, inn = S.shape
    ws = _ps_workspace(S, V, M, N)
    n = inn // M if which == 0 else out // V
    gain = np.zeros((n, n), dtype=np.int64)
    po, po_p = _host_perm(perm_out, out)
    pi, pi_p = _host_perm(perm_in, inn)
    _check(load_library().vnm_permutation_gain(_ptr(S), out, inn, S.stride(0), V, N, M, float(scale), which, slot,
                                               po_p, pi_p, gain.ctypes.data, _ptr(ws), ws.numel(), _stream(S)),
           "vnm_permutation_gain")
    return gain


def vnm_retained_score(S, V: int, M: int, scale: float, perm_out=None, perm_in=None, N: int = 2) -> int:
    """Objective of Eq. 7 at the given permutations (host int arrays or None)."""
    out, inn = S.shape
    ws = _ps_workspace(S, V, M, N)
    po, po_p = _host_perm(perm_out, out)
    pi, pi_p = _host_perm(perm_in, inn)
    tot = ctypes.c_int64(0)
    _check(load_library().vnm_retained_score(_ptr(S), out, inn, S.stride(0), V, N, M, float(scale), po_p, pi_p,
                                             ctypes.byref(tot), _ptr(ws), ws.numel(), _stream(S)),
           "vnm_retained_score")
    return tot.value


def vnm_lora_merge(W, B, A, scale: float, W_merged=None):
    """fp16(W + scale * B A) in the library's fixed fp32 order; W fp16 [out x in], B fp32 [out x r],
    A fp32 [r x in] (CUDA tensors)."""
    import torch
    assert W.is_cuda and W.dtype == torch.float16 and W.dim() == 2 and W.stride(1) == 1
    out, inn = W.shape
    r = B.shape[1]
    assert B.dtype == torch.float32 and A.dtype == torch.float32 and B.shape == (out, r) and A.shape == (r, inn)
    assert (r == 0) or (B.stride(1) == 1 and A.stride(1) == 1)
    if W_merged is None:
        W_merged = torch.empty_like(W)
    _check(load_library().vnm_lora_merge(_ptr(W), out, inn, W.stride(0), _ptr(B), B.stride(0) if r else 0, _ptr(A),
                                         A.stride(0) if r else inn, r, float(scale), _ptr(W_merged),
                                         W_merged.stride(0), _stream(W)), "vnm_lora_merge")
    return W_merged


def vnm_refresh_mask(W, B, A, scale: float, V: int, M: int, act=None, N: int = 2) -> Compressed:
    """Mask update of the LoRA stage with dynamic masks (Section 4.3): merge, score (RIA when `act`
    is given, else |w|), prune.  Returns the Compressed of the merged weight with its mask."""
    if act is None:
        return vnm_prune_compress(vnm_lora_merge(W, B, A, scale), V, M, N, want_mask=True)
    import torch
    assert W.is_cuda and W.dtype == torch.float16 and W.dim() == 2 and W.stride(1) == 1
    out, inn = W.shape
    r = B.shape[1]
    assert B.dtype == torch.float32 and A.dtype == torch.float32 and B.shape == (out, r) and A.shape == (r, inn)
    assert (r == 0) or (B.stride(1) == 1 and A.stride(1) == 1)
    assert act.is_cuda and act.dtype == torch.float32 and act.shape == (inn,) and act.is_contiguous()
    lib = load_library()
    b = ctypes.c_int64(0)
    _check(lib.vnm_refresh_mask_workspace_bytes(out, inn, V, N, M, ctypes.byref(b)), "vnm_refresh_mask_workspace_bytes")
    merged, c = torch.empty_like(W), None
    if b.value > 0:                     # three kernels without a score matrix, where sizes and alignment allow them
        values, meta, colidx, packed = _alloc(vnm_query_sizes(out, inn, V, M, N), W.device)
        mask = torch.empty((out, inn), dtype=torch.uint8, device=W.device)
        c = Compressed(values, meta, colidx, packed, out, inn, V, M, mask)
        ws = torch.empty(b.value, dtype=torch.uint8, device=W.device)
        status = lib.vnm_refresh_mask(
            _ptr(W), out, inn, W.stride(0), _ptr(B), B.stride(0) if r else 0, _ptr(A), A.stride(0) if r else inn, r,
            float(scale), _ptr(act), V, N, M, _ptr(merged), merged.stride(0), _ptr(values), _ptr(meta), _ptr(colidx),
            _ptr(mask), _ptr(packed), _ptr(ws), ws.numel(), _stream(W))
        if status == 0:
            return c
        del ws
        if status != 3:                 # rows that are not 16-byte aligned are the single steps' business
            _check(status, "vnm_refresh_mask")
    vnm_lora_merge(W, B, A, scale, merged)
    return vnm_prune_compress_scored(merged, vnm_ria_scores(merged, act), V, M, N, want_mask=True, out=c)


def vnm_stage_x(X, M: int, staged=None):
    """Re-lay X [T x in] for the matrix-core kernel; returns the staged uint8 tensor (reusable by
    every layer with the same `in` and M)."""
    import torch
    assert X.is_cuda and X.dtype == torch.float16 and X.dim() == 2 and X.stride(1) == 1
    T, inn = X.shape
    b = ctypes.c_int64(0)
    _check(load_library().vnm_stage_x_bytes(T, inn, M, ctypes.byref(b)), "vnm_stage_x_bytes")
    if staged is None:
        staged = torch.empty(max(b.value, 1), dtype=torch.uint8, device=X.device)
    _check(load_library().vnm_stage_x(_ptr(X), T, X.stride(0) if T > 0 else inn, inn, M, _ptr(staged),
                                      staged.numel(), _stream(X)), "vnm_stage_x")
    return staged


KERNEL_GENERIC, KERNEL_FEW_TOKENS, KERNEL_RESIDENT, KERNEL_STAGED = 0, 1, 2, 3


def vnm_spmm_kernel_choice(T: int, c: Compressed, workspace_bytes: int, N: int = 2) -> int:
    """Which kernel vnm_spmm runs for T tokens of this layer with a workspace of that size."""
    ch = ctypes.c_int(-1)
    _check(load_library().vnm_spmm_kernel_choice(T, c.out, c.inn, c.V, N, c.M, workspace_bytes, ctypes.byref(ch)),
           "vnm_spmm_kernel_choice")
    return ch.value


@functools.lru_cache(maxsize=1024, typed=True)      # (typed: 16.0 is refused, also after 16)
def vnm_spmm_scratch_bytes(T: int, out: int) -> int:
    b = ctypes.c_int64(0)
    _check(load_library().vnm_spmm_scratch_bytes(T, out, ctypes.byref(b)), "vnm_spmm_scratch_bytes")
    return b.value


def vnm_spmm_staged(staged, T: int, c: Compressed, N: int = 2, out_dtype=None, Y=None, scratch=None):
    """Y [T x out] from activations staged by vnm_stage_x and the packed weight of `c`.
    `scratch`: optional uint8 CUDA tensor for the split-K partial products (small T); by default
    the process-wide scratch tensor is used when vnm_spmm_scratch_bytes(T, out) > 0."""
    import torch
    if Y is None:
        Y = torch.empty((T, c.out), dtype=out_dtype or torch.float16, device=staged.device)
    y_dtype = {torch.float16: 0, torch.float32: 1}[Y.dtype]
    if scratch is None:
        nb = vnm_spmm_scratch_bytes(T, c.out)
        if nb > 0:
            scratch = _workspace((staged.device, "splitk"), nb)
    _check(load_library().vnm_spmm_staged(_ptr(staged), staged.numel(), T, _ptr(c.packed), c.out, c.inn, c.V, N, c.M, _ptr(Y),
                                          Y.stride(0) if T > 0 else c.out, y_dtype, _ptr(scratch),
                                          scratch.numel() if scratch is not None else 0, _stream(staged)),
           "vnm_spmm_staged")
    return Y


def vnm_decompress(c: Compressed, N: int = 2, W_out=None):
    import torch
    if W_out is None:
        W_out = torch.empty((c.out, c.inn), dtype=torch.float16, device=c.values.device)
    _check(load_library().vnm_decompress(_ptr(c.values), _ptr(c.meta), _ptr(c.colidx), c.out, c.inn, c.V, N,
                                         c.M, _ptr(W_out), W_out.stride(0), _stream(c.values)),
           "vnm_decompress")
    return W_out


def vnm_mask_diversity_log(V: int, M: int, N: int = 2) -> float:
    k = ctypes.c_double(0.0)
    _check(load_library().vnm_mask_diversity_log(V, N, M, ctypes.byref(k)), "vnm_mask_diversity_log")
    return k.value


def vnm_select_vm(candidates, threshold: float) -> int:
    """candidates: sequence of (V, M, speedup); returns the index of the selected one or -1."""
    n = len(candidates)
    V = (ctypes.c_int * max(n, 1))(*[int(c[0]) for c in candidates])
    M = (ctypes.c_int * max(n, 1))(*[int(c[1]) for c in candidates])
    sp = (ctypes.c_double * max(n, 1))(*[float(c[2]) for c in candidates])
    sel = ctypes.c_int(-1)
    _check(load_library().vnm_select_vm(V, M, sp, n, float(threshold), ctypes.byref(sel)), "vnm_select_vm")
    return sel.value


# --- layers in 8-bit integers and the norms between them ---------------------------------------------------------------

_DTYPES = None


def _dtype_code(dtype) -> int:
    """The vnm_dtype of a torch type; raises for one that the library does not take."""
    global _DTYPES
    if _DTYPES is None:
        import torch
        _DTYPES = {torch.float16: 0, torch.float32: 1, torch.bfloat16: 2}
    code = _DTYPES.get(dtype)
    if code is None:
        raise VnmError(3, f"unsupported V:N:M, dtype or path: {dtype}")
    return code


def _current_device() -> int:
    """The current CUDA device (torch's own query without its checks for a first use)."""
    global _current_device
    import torch
    _current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    return _current_device()


def _launch(what: str, fn, device, *args):
    """fn(*args, stream) on the device's current stream, with that device current."""
    if _current_device() == device.index:
        status = fn(*args, _raw_stream(device))
    else:
        import torch
        with torch.cuda.device(device):
            status = fn(*args, _raw_stream(device))
    if status:
        _check(status, what)


def _rows(name, t, T, n, device, dtype=None):
    """Checks a [T x n] tensor with rows of consecutive elements; returns its leading dimension."""
    assert t.shape == (T, n) and (dtype is None or t.dtype == dtype) and t.device == device, name
    if T > 1:
        ld, one = t.stride()
        assert ld >= n and (one == 1 or n == 1), name
        return ld
    assert T == 0 or n == 1 or t.stride(1) == 1, name
    return n


def _vector(name, t, n, device, dtype):
    if t is None:
        return 0
    assert t.shape == (n,) and t.dtype == dtype and t.device == device and t.is_contiguous(), name
    return t.data_ptr()


def _scratch(name, t, device):
    """The address of caller-supplied scratch memory, every byte of which the call may write."""
    import torch
    assert t.dtype == torch.uint8 and t.device == device and t.is_contiguous(), name
    return t.data_ptr()


def _empty_i8_rows(T: int, n: int, device):
    """int8 [T x n] with rows 16 bytes aligned, as the matrix-core kernels read them."""
    import torch
    ld = (n + 15) // 16 * 16
    q = torch.empty((T, ld), dtype=torch.int8, device=device)
    return q if ld == n else q[:, :n]


def vnm_quantize_x(X, Q=None, scale=None):
    """int8 activations with one scale per token: (Q int8 [T x n], scale fp32 [T]) of X [T x n] (fp16, bf16 or fp32),
    Q = rint(X * ((1 / max|X_t|) * 127)), scale = max|X_t| * (1 / 127).  A fresh Q has rows 16 bytes aligned."""
    import torch
    assert X.is_cuda and X.dim() == 2
    dev = X.device
    if _current_device() != dev.index:
        with torch.cuda.device(dev):
            return vnm_quantize_x(X, Q, scale)
    T, n = X.shape
    ldx = _rows("X", X, T, n, dev)
    if Q is None:
        ldq = (n + 15) // 16 * 16
        Q = torch.empty((T, ldq), dtype=torch.int8, device=dev)
        if ldq != n:
            Q = Q[:, :n]
    else:
        ldq = _rows("Q", Q, T, n, dev, torch.int8)
    if scale is None:
        scale = torch.empty(T, dtype=torch.float32, device=dev)
    else:
        _vector("scale", scale, T, dev, torch.float32)
    status = (_LIB or load_library()).vnm_quantize_x(X.data_ptr(), T, n, ldx, _dtype_code(X.dtype), Q.data_ptr(), ldq,
                                                     scale.data_ptr(), _raw_stream(dev))
    if status:
        _check(status, "vnm_quantize_x")
    return Q, scale


@dataclass
class CompressedI8:
    """A compressed layer in 8 bits (device tensors): int8 values in the order of Compressed.values, its positions and column
    indices, the opaque matrix-core copy, and one fp32 scale per output channel.  The products check types, sizes, layouts and
    devices of a layer once, and again after a field has been assigned."""
    values: object
    meta: object
    colidx: object
    packed: object
    scale: object
    out: int
    inn: int
    V: int
    M: int

    def __setattr__(self, name, value):
        self.__dict__["checked"] = False
        self.__dict__[name] = value


def _i8_packed_bytes(c: CompressedI8, N: int) -> int:
    b = ctypes.c_int64(0)
    _check(load_library().vnm_i8_packed_bytes(c.out, c.inn, c.V, N, c.M, ctypes.byref(b)), "vnm_i8_packed_bytes")
    return b.value


def _i8_packed(c: CompressedI8, N: int):
    import torch
    n = _i8_packed_bytes(c, N)
    return torch.empty(n, dtype=torch.uint8, device=c.values.device) if n > 0 else None


def _check_packed_i8(c: CompressedI8, nbytes: int):
    _scratch("packed", c.packed, c.values.device)
    assert c.packed.numel() >= nbytes, "packed"


def _check_layer_i8(c: CompressedI8, N: int):
    """What a product reads of a layer has the types, sizes and layouts that its kernels take, on the device of its values."""
    import torch
    s = vnm_query_sizes(c.out, c.inn, c.V, c.M, N)
    for name, t, dt, n in (("values", c.values, torch.int8, s.values_elems), ("meta", c.meta, torch.uint8, s.meta_bytes),
                           ("colidx", c.colidx, torch.uint8, s.colidx_bytes), ("scale", c.scale, torch.float32, c.out)):
        assert t.device == c.values.device and t.dtype == dt and t.is_contiguous() and t.numel() == n, name
    if c.packed is not None:
        _check_packed_i8(c, _i8_packed_bytes(c, N))
    c.__dict__["checked"] = True


def _check_triple(values, dtype, c, N):
    import torch
    s = vnm_query_sizes(c.out, c.inn, c.V, c.M, N)
    for name, t, dt, n in (("values", values, dtype, s.values_elems), ("meta", c.meta, torch.uint8, s.meta_bytes),
                           ("colidx", c.colidx, torch.uint8, s.colidx_bytes)):
        assert t.is_cuda and t.device == values.device and t.dtype == dt and t.is_contiguous() and t.numel() == n, name
    return s


def vnm_quantize_compressed(c: Compressed, N: int = 2) -> CompressedI8:
    """The layer's kept values in 8 bits, one scale per output channel; meta and colidx are shared with `c`."""
    import torch
    s = _check_triple(c.values, torch.float16, c, N)
    dev = c.values.device
    q = CompressedI8(torch.empty(s.values_elems, dtype=torch.int8, device=dev), c.meta, c.colidx, None,
                     torch.empty(c.out, dtype=torch.float32, device=dev), c.out, c.inn, c.V, c.M)
    q.packed = _i8_packed(q, N)
    _launch("vnm_quantize_compressed", load_library().vnm_quantize_compressed, dev, _ptr(c.values), _ptr(c.meta),
            _ptr(c.colidx), c.out, c.inn, c.V, N, c.M, _ptr(q.values), _ptr(q.scale), _ptr(q.packed))
    return q


def vnm_pack_i8(c: CompressedI8, N: int = 2) -> CompressedI8:
    """Fills c.packed from the triple (allocated where it is None and this V, M has one)."""
    import torch
    _check_triple(c.values, torch.int8, c, N)
    if c.packed is None:
        c.packed = _i8_packed(c, N)
    if c.packed is not None:
        n = _i8_packed_bytes(c, N)
        assert n > 0, "packed"
        _check_packed_i8(c, n)
        _launch("vnm_pack_i8", load_library().vnm_pack_i8, c.values.device, _ptr(c.values), _ptr(c.meta), _ptr(c.colidx), c.out,
                c.inn, c.V, N, c.M, _ptr(c.packed))
    return c


@functools.lru_cache(maxsize=1024, typed=True)      # (typed: 16.0 is refused, also after 16)
def _spmm_i8_workspace_bytes(T: int, out: int, inn: int, V: int, N: int, M: int) -> int:
    b = ctypes.c_int64(0)
    _check(load_library().vnm_spmm_i8_workspace_bytes(T, out, inn, V, N, M, ctypes.byref(b)), "vnm_spmm_i8_workspace_bytes")
    return b.value


def vnm_spmm_i8_workspace_bytes(T: int, c: CompressedI8, N: int = 2) -> int:
    return _spmm_i8_workspace_bytes(T, c.out, c.inn, c.V, N, c.M)


_I8_MAX_ROW_PITCH = 1 << 24                          # of activations that the matrix-core kernels read


def vnm_spmm_i8(Q, scale, c: CompressedI8, bias=None, N: int = 2, out_dtype=None, path: int = PATH_AUTO, Y=None, workspace=None):
    """Y [T x out] = (Q . Wq^T) * c.scale[o] * scale[t] + bias[o], sums exact in int32, Y in fp16, bf16 or fp32 (default fp16).
    Q, scale as vnm_quantize_x leaves them, `bias` fp16 [out].  Rows of Q that are not 16-byte aligned, and layers without a packed
    copy (V = 16, M > 16), are served by a kernel that is slow on many tokens.  `workspace`: optional uint8 CUDA tensor of at least
    vnm_spmm_i8_workspace_bytes(T, c) bytes; by default the call takes one from torch's allocator."""
    import torch
    assert Q.is_cuda and Q.dim() == 2
    dev = Q.device
    if _current_device() != dev.index:
        with torch.cuda.device(dev):
            return vnm_spmm_i8(Q, scale, c, bias, N, out_dtype, path, Y, workspace)
    T, inn = Q.shape
    if not c.checked:
        _check_layer_i8(c, N)
    out, packed = c.out, c.packed
    assert inn == c.inn and c.values.device == dev
    ldq = _rows("Q", Q, T, inn, dev, torch.int8)
    if T == 1:
        ldq = (inn + 15) // 16 * 16              # (one row: whatever the view's stride)
    if Y is None:
        Y, ldy = torch.empty((T, out), dtype=out_dtype or torch.float16, device=dev), out
    else:
        ldy = _rows("Y", Y, T, out, dev)
    at = Q.data_ptr()
    if workspace is None and packed is not None and path != PATH_GENERIC:
        need = _spmm_i8_workspace_bytes(T, out, inn, c.V, N, c.M)
        if need and at % 16 == 0 and ldq % 16 == 0 and ldq <= _I8_MAX_ROW_PITCH:    # (else the kernel on the triple serves the call)
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    status = (_LIB or load_library()).vnm_spmm_i8(
        at, T, ldq, _vector("scale", scale, T, dev, torch.float32), c.values.data_ptr(), c.meta.data_ptr(),
        c.colidx.data_ptr(), 0 if packed is None else packed.data_ptr(), c.scale.data_ptr(), out, inn, c.V, N, c.M,
        _vector("bias", bias, out, dev, torch.float16), Y.data_ptr(), ldy, _dtype_code(Y.dtype), path,
        0 if workspace is None else _scratch("workspace", workspace, dev), 0 if workspace is None else workspace.numel(), _raw_stream(dev))
    if status:
        _check(status, "vnm_spmm_i8")
    return Y


def vnm_stage_q(Q, M: int, staged=None):
    """Re-lay int8 activations Q [T x in] for the many-token kernel; returns the staged uint8 tensor (reusable by every int8 layer
    with the same `in` and M)."""
    import torch
    assert Q.is_cuda and Q.dim() == 2
    T, inn = Q.shape
    dev = Q.device
    ldq = _rows("Q", Q, T, inn, dev, torch.int8)
    if T <= 1:
        ldq = (inn + 15) // 16 * 16              # (one row: whatever the view's stride)
    b = ctypes.c_int64(0)
    _check(load_library().vnm_stage_q_bytes(T, inn, M, ctypes.byref(b)), "vnm_stage_q_bytes")
    if staged is None:
        staged = torch.empty(max(b.value, 1), dtype=torch.uint8, device=dev)
    _launch("vnm_stage_q", load_library().vnm_stage_q, dev, Q.data_ptr(), T, ldq, inn, M, _scratch("staged", staged, dev), staged.numel())
    return staged


def vnm_spmm_i8_staged(staged, scale, c: CompressedI8, bias=None, N: int = 2, out_dtype=None, Y=None):
    """vnm_spmm_i8 on activations staged by vnm_stage_q; `scale` fp32 [T] as there."""
    import torch
    dev, T = staged.device, scale.shape[0]
    if not c.checked:
        _check_layer_i8(c, N)
    assert staged.is_cuda and c.packed is not None and c.values.device == dev
    if Y is None:
        Y = torch.empty((T, c.out), dtype=out_dtype or torch.float16, device=dev)
    ldy = _rows("Y", Y, T, c.out, dev)
    _launch("vnm_spmm_i8_staged", load_library().vnm_spmm_i8_staged, dev, _scratch("staged", staged, dev), staged.numel(), T,
            _vector("scale", scale, T, dev, torch.float32), c.packed.data_ptr(), c.scale.data_ptr(), c.out, c.inn, c.V, N, c.M,
            _vector("bias", bias, c.out, dev, torch.float16), Y.data_ptr(), ldy, _dtype_code(Y.dtype))
    return Y


_NORMS = {"none": 0, "rms": 1, "layer": 2}


class ResidualNorm(NamedTuple):
    """What vnm_residual_norm returns: the new residual stream, the normalised rows (or their int8 values with `scale`), and
    the statistics that vnm_residual_norm_backward takes."""
    h: object
    x: object
    scale: object
    stats: object


class ResidualNormGrads(NamedTuple):
    h: object
    y: object
    gate: object
    post_weight: object
    post_bias: object
    pre_weight: object
    pre_bias: object


def _norm_operands(h, y, gate, gate_tokens, x_dtype, vectors):
    """Shared checks of the two norm calls: (T, n, device, x type, leading dimensions of h, y and gate)."""
    assert h.is_cuda and h.dim() == 2
    T, n = h.shape
    dev = h.device
    if x_dtype is None:
        x_dtype = y.dtype if y is not None else next((t.dtype for t in vectors if t is not None), h.dtype)
    ldh = _rows("h", h, T, n, dev)
    ldy = 0 if y is None else _rows("y", y, T, n, dev, x_dtype)
    ldg = 0
    if gate is not None:
        assert gate_tokens >= 0, "gate_tokens"
        if gate_tokens == 0:
            _vector("gate", gate, n, dev, x_dtype)
        else:
            ldg = _rows("gate", gate, -(-T // gate_tokens), n, dev, x_dtype)
    return T, n, dev, x_dtype, ldh, ldy, ldg


def vnm_residual_norm(h, y=None, gate=None, gate_tokens: int = 0, residual_scale: float = 1.0, post: str = "none",
                      post_weight=None, post_bias=None, post_eps: float = 1e-5, pre: str = "none", pre_weight=None,
                      pre_bias=None, pre_eps: float = 1e-5, x_dtype=None, int8: bool = False, want_x: bool = True,
                      want_stats: bool = False, h_out=None) -> ResidualNorm:
    """Between two blocks: h' = residual_scale * h + gate * norm_post(y), x = norm_pre(h').

    h [T x n] is the residual stream (type of y, or fp32), y [T x n] the block's output (None: only h).  `gate`: [n], or with
    gate_tokens > 0 one row per that many tokens.  post, pre: "none", "rms" or "layer".  Weights, biases and gate have y's type,
    which is x's too (`x_dtype` where there is none of them).  int8: x leaves as int8 rows with a scale per token, ready for
    vnm_spmm_i8.  h_out: a tensor for h' (h itself: in place); a fresh one by default."""
    import torch
    T, n, dev, xt, ldh, ldy, ldg = _norm_operands(h, y, gate, gate_tokens, x_dtype, (post_weight, post_bias, pre_weight, pre_bias))
    if h_out is None:
        h_out, ldho = torch.empty((T, n), dtype=h.dtype, device=dev), n
    else:
        ldho = _rows("h_out", h_out, T, n, dev, h.dtype)
    x = q = scale = stats = None
    if want_x and int8:
        q, scale = _empty_i8_rows(T, n, dev), torch.empty(T, dtype=torch.float32, device=dev)
    elif want_x:
        x = torch.empty((T, n), dtype=xt, device=dev)
    if want_stats:
        stats = torch.empty((T, 4), dtype=torch.float32, device=dev)
    a = _NORM_ARGS.pack(
        T, n, _dtype_code(h.dtype), _dtype_code(xt), _NORMS[post], _NORMS[pre], post_eps, pre_eps, residual_scale, gate_tokens,
        h.data_ptr(), _ptr(y), _ptr(gate), _vector("post_weight", post_weight, n, dev, xt), _vector("post_bias", post_bias, n, dev, xt),
        _vector("pre_weight", pre_weight, n, dev, xt), _vector("pre_bias", pre_bias, n, dev, xt), ldh, ldy, ldg,
        h_out.data_ptr(), _ptr(x), _ptr(q), _ptr(scale), _ptr(stats), ldho, n, (n + 15) // 16 * 16)
    _launch("vnm_residual_norm", load_library().vnm_residual_norm, dev, a)
    return ResidualNorm(h_out, q if int8 else x, scale, stats)


def vnm_residual_norm_backward(h, stats, dx=None, dh=None, y=None, gate=None, gate_tokens: int = 0, residual_scale: float = 1.0,
                               post: str = "none", post_weight=None, post_bias=None, pre: str = "none", pre_weight=None,
                               pre_bias=None, want_dh: bool = True, want_dy: bool = True, want_params: bool = True,
                               workspace=None) -> ResidualNormGrads:
    """Gradients of vnm_residual_norm from dx and dh, those of its results x and h (either may be None).  `h` and `stats` are
    what the forward call returned (its h, with want_stats), everything else what it was given.  Sums over the tokens (weights,
    biases, gate) come in fp32; the gradient of an argument that is None is None, and without dx those of the pre norm's are too."""
    import torch
    T, n, dev, xt, ldh, ldy, ldg = _norm_operands(h, y, gate, gate_tokens, None if dx is None else dx.dtype,
                                                  (post_weight, post_bias, pre_weight, pre_bias, gate))
    lddx = 0 if dx is None else _rows("dx", dx, T, n, dev, xt)
    lddho = 0 if dh is None else _rows("dh", dh, T, n, dev, h.dtype)
    assert stats is None or (stats.shape == (T, 4) and stats.dtype == torch.float32 and stats.is_contiguous() and stats.device == dev)
    gh = torch.empty((T, n), dtype=h.dtype, device=dev) if want_dh else None
    gy = torch.empty((T, n), dtype=xt, device=dev) if want_dy and y is not None else None
    _vector("pre_bias", pre_bias, n, dev, xt)
    g_gate = g_ow = g_ob = g_pw = g_pb = None
    lib, tokens = load_library(), gate_tokens if gate is not None else 0
    if want_params:
        g_gate = torch.empty(gate.shape, dtype=torch.float32, device=dev) if gate is not None else None
        through = (post_weight, post_bias) + ((pre_weight, pre_bias) if dx is not None else (None, None))
        count = sum(t is not None for t in through)
        if count:
            rows = iter(torch.empty((count, n), dtype=torch.float32, device=dev).unbind(0))
            g_ow, g_ob, g_pw, g_pb = (None if t is None else next(rows) for t in through)
        if workspace is None and (count or gate is not None):
            workspace = torch.empty(_backward_workspace_bytes(T, n, tokens), dtype=torch.uint8, device=dev)
    a = _NORM_BACKWARD_ARGS.pack(
        T, n, _dtype_code(h.dtype), _dtype_code(xt), _NORMS[post], _NORMS[pre], residual_scale, tokens,
        _ptr(dx), _ptr(dh), h.data_ptr(), _ptr(y), _ptr(gate), _vector("post_weight", post_weight, n, dev, xt),
        _vector("post_bias", post_bias, n, dev, xt), _vector("pre_weight", pre_weight, n, dev, xt), _ptr(stats), lddx, lddho, ldh, ldy,
        ldg, _ptr(gh), _ptr(gy), _ptr(g_ow), _ptr(g_ob), _ptr(g_pw), _ptr(g_pb), _ptr(g_gate), n, n)
    _launch("vnm_residual_norm_backward", lib.vnm_residual_norm_backward, dev, a,
            0 if workspace is None else _scratch("workspace", workspace, dev), 0 if workspace is None else workspace.numel())
    return ResidualNormGrads(gh, gy, g_gate, g_ow, g_ob, g_pw, g_pb)


@functools.lru_cache(maxsize=1024, typed=True)      # (typed: 16.0 is refused, also after 16)
def _backward_workspace_bytes(T: int, n: int, gate_tokens: int) -> int:
    b = ctypes.c_int64(0)
    _check(load_library().vnm_residual_norm_backward_workspace_bytes(T, n, gate_tokens, ctypes.byref(b)),
           "vnm_residual_norm_backward_workspace_bytes")
    return b.value
