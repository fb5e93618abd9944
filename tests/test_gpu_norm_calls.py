"""Calls of the norms that a program may make and that test_gpu_residual_norm.py does not: rows of other strides in the backward
pass, a gate row per token, more gate rows than a grid has rows, more tokens than workgroups, two threads at once, and a captured
pass with other inputs in every replay."""

import threading

import pytest
import torch

import paper_2410_16135_amd as vnm
from tests.test_gpu_residual_norm import DEV, EPS, U, backward_plain, make, on, plain, within

pytestmark = pytest.mark.gpu


def strided(t, ld, first):
    """The same values in rows ld apart, `first` elements into memory that holds sevens."""
    buf = torch.full(((t.shape[0] + 1) * ld + first,), 7.0, dtype=t.dtype, device=t.device)
    view = buf.as_strided(t.shape, (ld, 1), first)
    view.copy_(t)
    return view


@pytest.mark.parametrize("n", [64, 200, 513, 1024])
@pytest.mark.parametrize("h,x", [("fp32", "bf16"), ("fp16", "fp16")])
def test_backward_of_strided_rows(n, h, x):
    """Aligned or not, the same arithmetic: equal bits."""
    T, gate = 21, 4
    t = on(make(T, n, h, x, "layer", "rms", gate))
    kw = dict(gate_tokens=gate, residual_scale=0.5, pre="layer", post="rms")
    f = vnm.vnm_residual_norm(**t, **kw, want_stats=True)
    g = torch.Generator(device=DEV).manual_seed(1)
    dx = torch.randn(T, n, generator=g, device=DEV).to(t["y"].dtype)
    dh = torch.randn(T, n, generator=g, device=DEV).to(t["h"].dtype)
    want = vnm.vnm_residual_norm_backward(**{**t, "h": f.h}, stats=f.stats, dx=dx, dh=dh, **kw)
    for ld, first in ((-(-n // 8) * 8 + 16, 8), (n + 3, 1)):
        s = {**t, "h": strided(f.h, ld, first), "y": strided(t["y"], ld, first), "gate": strided(t["gate"], ld, first)}
        got = vnm.vnm_residual_norm_backward(**s, stats=f.stats, dx=strided(dx, ld, first), dh=strided(dh, ld, first), **kw)
        assert all(a is None and b is None or torch.equal(a, b) for a, b in zip(got, want)), (ld, first)
        # and the forward pass into rows of its own stride
        out = strided(torch.zeros_like(f.h), ld + 5, 3)
        r = vnm.vnm_residual_norm(**{**t, "y": s["y"], "gate": s["gate"], "h": strided(t["h"], ld, first)}, **kw, want_stats=True, h_out=out)
        assert r.h is out and torch.equal(out, f.h) and torch.equal(r.x, f.x) and torch.equal(r.stats, f.stats)


@pytest.mark.parametrize("T,n,gate", [(70001, 8, 1), (140003, 16, 2), (5000, 64, 1), (9, 4104, 1), (7, 40, 100)])
def test_many_gate_rows(T, n, gate):
    """A gate row per token or two, more of them than 65535; a gate row that has more tokens than there are."""
    pre, post = "rms", "none"
    t = make(T, n, "fp32", "fp16", pre, post, gate)
    s = on(t)
    f = vnm.vnm_residual_norm(**s, gate_tokens=gate, pre=pre, post=post, want_stats=True)
    h64, x64, _, mh, mx = plain(t, gate, 1.0, pre, post)
    assert within(f.h, h64, EPS["fp32"] * h64.abs() + 64 * U * mh) is True
    assert within(f.x, x64, EPS["fp16"] * x64.abs() + 192 * U * mx + 2.0 ** -25) is True
    g = torch.Generator().manual_seed(5)
    dx, dh = torch.randn(T, n, generator=g).half(), torch.randn(T, n, generator=g)
    b = vnm.vnm_residual_norm_backward(**{**s, "h": f.h}, stats=f.stats, dx=dx.to(DEV), dh=dh.to(DEV), gate_tokens=gate, pre=pre, post=post)
    want, mag = backward_plain(t, f.h.double().cpu(), f.stats.cpu(), dx.double(), dh.double(), gate, 1.0, pre, post)
    # the roundings of test_backward: 256 of the terms, and for sums one more per token that is added
    for name, count in (("gate", gate), ("pre_weight", T), ("h", 0), ("y", 0)):
        got = getattr(b, name)
        eps = EPS["fp16"] if name == "y" else EPS["fp32"] if name == "h" else 0.0
        tol = eps * want[name].abs() + (256 + count) * U * mag[name] + (2.0 ** -25 if name == "y" else 0.0) + 1e-35
        assert within(got.view(want[name].shape), want[name], tol) is True, name


def test_two_threads_at_once():
    """Each on a stream of its own, from the first call on."""
    T, n = 600, 768
    t = on(make(T, n, "fp32", "bf16", "layer", "rms", 50))
    kw = dict(pre="layer", post="rms", gate_tokens=50)
    dx, dh = torch.randn(T, n, device=DEV).bfloat16(), torch.randn(T, n, device=DEV)
    torch.cuda.synchronize()
    got = [None, None]

    def work(k):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                f = vnm.vnm_residual_norm(**t, **kw, want_stats=True)
                q, s = vnm.vnm_quantize_x(f.x)
                b = vnm.vnm_residual_norm_backward(**{**t, "h": f.h}, stats=f.stats, dx=dx, dh=dh, **kw)
            torch.cuda.current_stream().synchronize()
            got[k] = [*f, q, s, *b]

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert all(a is None and b is None or torch.equal(a, b) for a, b in zip(*got))


def test_captured_quantizer_and_norm():
    """Two graphs of the quantizer, the norm with an int8 result and the backward pass, replayed in turn with other inputs."""
    T, n = 130, 1024
    t = on(make(T, n, "fp16", "fp16", "rms", "layer", -1))
    kw = dict(pre="rms", post="layer")
    dx = torch.empty(T, n, dtype=torch.float16, device=DEV)

    def call():
        f = vnm.vnm_residual_norm(**t, **kw, want_stats=True)
        i = vnm.vnm_residual_norm(**t, **kw, int8=True, want_stats=True)
        b = vnm.vnm_residual_norm_backward(**{**t, "h": f.h}, stats=f.stats, dx=dx, **kw)
        return [*f, *i, *b, *vnm.vnm_quantize_x(f.h)]

    dx.zero_()
    call()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = call()
        graphs.append((g, out))
    gen = torch.Generator(device=DEV).manual_seed(3)
    for _ in range(4):
        dx.copy_(torch.randn(T, n, generator=gen, device=DEV))
        t["h"].copy_(torch.randn(T, n, generator=gen, device=DEV))
        t["y"].copy_(torch.randn(T, n, generator=gen, device=DEV))
        for g, _ in graphs:
            g.replay()
        eager = call()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(a is None and b is None or torch.equal(a, b) for a, b in zip(out, eager))
