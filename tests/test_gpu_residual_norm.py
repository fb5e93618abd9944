"""The norms between two blocks and their gradients on the GPU, against plain forms in float64.

Tolerances.  A result differs from the plain form by its own rounding, eps / 2 of its type (2^-11, 2^-8, 2^-24), and by the errors of
the fp32 arithmetic behind it.  A sum over a row is at most 16 additions per thread, 6 in a wave and 16 between waves, so at most
about 40 roundings of 2^-24 relative to the sum of the magnitudes, which a square root halves; with the few operations before and
after it 64 roundings of the terms behind h', and three times as many (two norms, one through the other) behind x, bound the rest.
`mag` is the size of those terms (int8_reference.norm_magnitude).  2^-25 is half of fp16's smallest step, 2^-24, by which results
below its normal range are rounded."""

import numpy as np
import pytest
import torch

import paper_2410_16135_amd as vnm
from tests import int8_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
U = 2.0 ** -24


def make(T, n, h, x, pre, post, gate=0, y=True, seed=0):
    g = torch.Generator().manual_seed(seed + 31 * T + n)
    rnd = lambda *s: torch.randn(*s, generator=g)
    xt = ref.TYPES[x]
    t = {"h": (3 * rnd(T, n) + 0.5).to(ref.TYPES[h]), "y": rnd(T, n).to(xt) if y else None, "gate": None}
    for which, kind in (("pre", pre), ("post", post)):
        t[which + "_weight"] = (1 + 0.2 * rnd(n)).to(xt) if kind != "none" else None
        t[which + "_bias"] = (0.3 * rnd(n)).to(xt) if kind == "layer" else None
    if gate:
        rows = 1 if gate < 0 else -(-T // gate)
        t["gate"] = rnd(n).to(xt) if gate < 0 else rnd(rows, n).to(xt)
    return t


def d64(t):
    return None if t is None else t.double()


def on(t):
    return {k: None if v is None else v.to(DEV) for k, v in t.items()}


def gate_rows(t, gate, T):
    return None if t["gate"] is None else d64(t["gate"])[None].expand(T, -1) if gate < 0 else d64(t["gate"]).repeat_interleave(gate, 0)[:T]


def plain(t, gate, scale, pre, post, eps=1e-5):
    return ref.residual_norm(d64(t["h"]), d64(t["y"]), gate_rows(t, gate, t["h"].shape[0]), scale,
                             (post, d64(t["post_weight"]), d64(t["post_bias"]), eps), (pre, d64(t["pre_weight"]), d64(t["pre_bias"]), eps))


def within(got, want, tol):
    got = got.double().cpu()
    bad = ~((got - want).abs() <= tol)
    return not bool(bad.any()) or f"{int(bad.sum())} off, worst {float(((got - want).abs() / tol).max()):.3g} of the tolerance"


WIDTHS = [1, 2, 7, 64, 100, 384, 512, 513, 768, 1024, 1030, 2048, 2056, 4096, 5001, 8192, 11008, 16384]
KINDS = [("rms", "none"), ("layer", "none"), ("rms", "rms"), ("layer", "layer"), ("none", "layer"), ("rms", "layer")]


@pytest.mark.parametrize("h,x", [("fp16", "fp16"), ("bf16", "bf16"), ("fp32", "fp16"), ("fp32", "bf16"), ("fp32", "fp32")])
@pytest.mark.parametrize("n", WIDTHS)
def test_forward(n, h, x):
    pre, post = KINDS[WIDTHS.index(n) % len(KINDS)]
    for T, gate, scale in ((1, 0, 1.0), (5, -1, 0.5), (11, 4, 1.0)):
        t = make(T, n, h, x, pre, post, gate)
        r = vnm.vnm_residual_norm(**on(t), gate_tokens=max(gate, 0), residual_scale=scale, pre=pre, post=post, want_stats=True)
        h64, x64, stats, mh, mx = plain(t, gate, scale, pre, post)
        assert within(r.h, h64, EPS[h] * h64.abs() + 64 * U * mh + 2.0 ** -25) is True
        assert within(r.x, x64, EPS[x] * x64.abs() + 192 * U * mx + 2.0 ** -25) is True
        assert r.h.dtype == ref.TYPES[h] and r.x.dtype == ref.TYPES[x]
        # reciprocal deviations to 192 roundings of what is under the root; means to as many of the terms
        spread = mh.square().mean(1, keepdim=True).sqrt() * stats[:, 3:4]
        assert within(r.stats[:, 3:4], stats[:, 3:4], 192 * U * (1 + spread) * stats[:, 3:4]) is True
        assert within(r.stats[:, 2:3], stats[:, 2:3], 64 * U * mh.mean(1, keepdim=True) + 1e-30) is True


@pytest.mark.parametrize("n,pre,post", [(64, "rms", "none"), (513, "layer", "rms"), (4096, "rms", "rms"), (8200, "none", "none"), (16384, "layer", "none")])
def test_forward_int8(n, pre, post):
    t = make(9, n, "fp32", "bf16", pre, post, 2)
    r = vnm.vnm_residual_norm(**on(t), gate_tokens=2, pre=pre, post=post, int8=True)
    _, x64, _, _, mx = plain(t, 2, 1.0, pre, post)
    top = x64.abs().amax(1, keepdim=True)
    err = 192 * U * (mx + mx.amax(1, keepdim=True))               # of a value, and of the row's largest
    assert within(r.scale[:, None], top / 127, err.amax(1, keepdim=True) / 127 + U * top / 127) is True
    # a value stands within half a step of the exact one
    assert within(r.x.double().cpu() * r.scale.double().cpu()[:, None], x64, (0.5 + 1e-5) * top / 127 + 2 * err) is True
    assert int(r.x.cpu().int().abs().max()) == 127


def test_forward_in_place_and_strides():
    t = on(make(7, 200, "fp16", "fp16", "layer", "none", -1))
    want = vnm.vnm_residual_norm(**t, pre="layer", residual_scale=0.5)
    # rows of other strides and alignments
    for ld, first in ((208, 0), (216, 8), (203, 1)):
        s = dict(t)
        for name in ("h", "y"):
            buf = torch.full((9, ld + 16), 7.0, dtype=torch.float16, device=DEV)
            buf[1:8, first:first + 200] = t[name]
            s[name] = buf[1:8, first:first + 200]
            s[name + "_buf"] = buf
        hb, yb = s.pop("h_buf"), s.pop("y_buf")
        r = vnm.vnm_residual_norm(**s, pre="layer", residual_scale=0.5, h_out=s["h"])
        assert torch.equal(r.x, want.x) and torch.equal(s["h"], want.h)
        s["h"].fill_(7.0)
        assert bool((hb == 7.0).all())                            # around the rows nothing was written
        assert torch.equal(yb[1:8, first:first + 200], t["y"])
    r = vnm.vnm_residual_norm(**t, pre="layer", residual_scale=0.5, want_x=False)
    assert r.x is None and torch.equal(r.h, want.h)


def test_forward_h_only_and_degenerate_rows():
    # without a block's output: only the norm; rows of zeros, of one value, and of values that are not numbers
    h = torch.zeros(6, 96)
    h[1] = 2.5
    h[2, 5] = float("inf")
    h[3, 7] = float("nan")
    h[4, 0] = 1e30                                                # its square leaves fp32: r is 0
    h[5, 3] = 1.0
    r = vnm.vnm_residual_norm(h.to(DEV), pre="layer", x_dtype=torch.float32)
    assert torch.equal(torch.nan_to_num(r.h.cpu(), nan=9.0), torch.nan_to_num(h, nan=9.0))
    x = r.x.cpu()
    assert bool((x[0] == 0).all()) and bool((x[1] == 0).all())
    assert bool(torch.isnan(x[2]).all()) and bool(torch.isnan(x[3]).all()) and not bool(torch.isnan(x[5]).any())
    q = vnm.vnm_residual_norm(h.to(DEV), pre="layer", x_dtype=torch.float32, int8=True)
    assert q.scale.cpu()[0] == 0 and q.scale.cpu()[1] == 0 and torch.isnan(q.scale.cpu()[2:4]).all()
    assert bool((q.x.cpu()[:4] == 0).all()) and int(q.x.cpu()[5].abs().max()) == 127
    assert vnm.vnm_residual_norm(torch.empty(0, 96, device=DEV), pre="rms").x.shape == (0, 96)


def test_forward_large_mean():
    # a mean that is 1000 deviations away: the variance is a sum of squared deviations and does not cancel
    g = torch.Generator().manual_seed(1)
    h = 1000 + torch.randn(3, 4096, generator=g)
    r = vnm.vnm_residual_norm(h.to(DEV), pre="layer", x_dtype=torch.float32)
    x64 = ref.normed(h.double(), "layer", None, None, 1e-5)[0]
    # the mean is off by at most 40 roundings of 1000, every other error is smaller
    assert within(r.x, x64, 64 * U * 1000 * torch.ones_like(x64)) is True


def test_many_rows():
    # more rows than workgroups: every one is written
    t = make(20011, 64, "fp16", "fp16", "rms", "none", 7)
    r = vnm.vnm_residual_norm(**on(t), gate_tokens=7, pre="rms")
    h64, x64, _, mh, mx = plain(t, 7, 1.0, "rms", "none")
    assert within(r.h, h64, EPS["fp16"] * h64.abs() + 64 * U * mh) is True
    assert within(r.x, x64, EPS["fp16"] * x64.abs() + 192 * U * mx + 2.0 ** -25) is True


# --- gradients --------------------------------------------------------------------------------------------------------

def backward_plain(t, h_new, stats, dx, dh, gate, scale, pre, post):
    """The formulas in float64 on the stored rows and statistics; and for every result a bound of the terms behind it."""
    T, n = h_new.shape
    ym, yr, hm, hr = stats.double().unbind(1)
    out, mag = {}, {}

    def through(g, gm, xhat, r, kind):
        s1, s2 = (g * xhat).mean(1, keepdim=True), (g.mean(1, keepdim=True) if kind == "layer" else 0.0)
        m = gm + xhat.abs() * (gm * xhat.abs()).mean(1, keepdim=True) + gm.mean(1, keepdim=True)
        return r[:, None] * (g - s2 - xhat * s1), r[:, None] * m

    d, m = dh, dh.abs()
    if pre != "none":
        xhat = (h_new - hm[:, None]) * hr[:, None]
        xm = (h_new.abs() + hm[:, None].abs()) * hr[:, None]         # what is behind xhat
        w = d64(t["pre_weight"])
        out["pre_weight"], mag["pre_weight"] = (dx * xhat).sum(0), (dx.abs() * xm).sum(0)
        out["pre_bias"], mag["pre_bias"] = dx.sum(0), dx.abs().sum(0)
        a, am = through(dx * w, (dx * w).abs(), xhat, hr, pre)
        am = am + hr[:, None] * (xm * (dx * w * xhat).abs().mean(1, keepdim=True) + xhat.abs() * ((dx * w).abs() * xm).mean(1, keepdim=True))
        d, m = d + a, m + am
    else:
        d, m = d + dx, m + dx.abs()
    out["h"], mag["h"] = scale * d, abs(scale) * m
    yhat = (d64(t["y"]) - ym[:, None]) * yr[:, None]
    yhm = (d64(t["y"]).abs() + ym[:, None].abs()) * yr[:, None]
    ow = 1.0 if t["post_weight"] is None else d64(t["post_weight"])
    ob = 0.0 if t["post_bias"] is None else d64(t["post_bias"])
    rows = gate_rows(t, gate, T)
    if rows is not None:
        p, pm = yhat * ow + ob, yhm * abs(ow) + abs(ob)
        groups = torch.zeros(T, dtype=torch.long) if gate < 0 else torch.arange(T) // gate
        count = int(groups[-1]) + 1
        out["gate"] = torch.zeros(count, n, dtype=torch.float64).index_add_(0, groups, d * p)
        mag["gate"] = torch.zeros(count, n, dtype=torch.float64).index_add_(0, groups, m * pm)
        d, m = d * rows, m * rows.abs()
    if post != "none":
        out["post_weight"], mag["post_weight"] = (d * yhat).sum(0), (m * yhm).sum(0)
        out["post_bias"], mag["post_bias"] = d.sum(0), m.sum(0)
        g, gm = d * ow, m * abs(ow)
        d, m2 = through(g, gm, yhat, yr, post)
        m = m2 + yr[:, None] * (yhm * (gm * yhat.abs()).mean(1, keepdim=True) + yhat.abs() * (gm * yhm).mean(1, keepdim=True))
    out["y"], mag["y"] = d, m
    return out, mag


BACK_WIDTHS = [1, 7, 64, 384, 513, 768, 1024, 1500, 2048, 4096, 4100, 8192, 8200, 16384]


@pytest.mark.parametrize("h,x", [("fp16", "fp16"), ("bf16", "bf16"), ("fp32", "fp16"), ("fp32", "bf16"), ("fp32", "fp32")])
@pytest.mark.parametrize("n", BACK_WIDTHS)
def test_backward(n, h, x):
    pre, post = KINDS[BACK_WIDTHS.index(n) % len(KINDS)]
    for T, gate, scale in ((1, -1, 1.0), (13, 5, 0.5), (300 if n < 2000 else 40, 0, 1.0), (900 if n < 600 else 30, 7, 1.0)):
        t = make(T, n, h, x, pre, post, gate)
        s = on(t)
        f = vnm.vnm_residual_norm(**s, gate_tokens=max(gate, 0), residual_scale=scale, pre=pre, post=post, want_stats=True)
        g = torch.Generator().manual_seed(5)
        dx, dh = torch.randn(T, n, generator=g).to(ref.TYPES[x]), torch.randn(T, n, generator=g).to(ref.TYPES[h])
        s["h"] = f.h
        b = vnm.vnm_residual_norm_backward(stats=f.stats, dx=dx.to(DEV), dh=dh.to(DEV), gate_tokens=max(gate, 0), residual_scale=scale,
                                           pre=pre, post=post, **s)
        want, mag = backward_plain(t, f.h.double().cpu(), f.stats.cpu(), dx.double(), dh.double(), gate, scale, pre, post)
        # as many roundings as in the forward pass, and for the sums over the tokens one more per token in a worker's run and per worker
        for name, got in b._asdict().items():
            if got is None:
                assert name not in ("h", "y")
                continue
            sums = name not in ("h", "y")
            eps = 0.0 if sums else EPS[h] if name == "h" else EPS[x]
            tol = eps * want[name].abs() + (256 + (T if sums else 0)) * U * mag[name] + 2.0 ** -25 * (not sums) + 1e-35
            assert within(got.view(want[name].shape), want[name], tol) is True, (name, T)
            assert got.dtype == (torch.float32 if sums else ref.TYPES[h] if name == "h" else ref.TYPES[x])
        assert (b.gate is None) == (gate == 0) and (b.post_weight is None) == (post == "none")


@pytest.mark.parametrize("pre,post", [("rms", "rms"), ("layer", "layer"), ("layer", "none"), ("none", "rms")])
def test_backward_against_differences(pre, post):
    """d/ds of a fixed linear function of both results along a direction of every input, by central differences of the forward pass.
    With steps of 2^-6 of rows whose deviation is about 3 the truncation (a sixth of the step's square times the third derivative, whose
    size per unit of the norms' inputs is of order 1) is below 1e-3 of the terms' root sum of squares, and fp32 roundings of 2^-24
    divided by the step are smaller."""
    T, n, gate = 6, 96, 2
    t = on(make(T, n, "fp32", "fp32", pre, post, gate, seed=4))
    kw = dict(gate_tokens=gate, residual_scale=0.75, pre=pre, post=post)
    g = torch.Generator().manual_seed(9)
    cx, ch = torch.randn(T, n, generator=g).to(DEV), torch.randn(T, n, generator=g).to(DEV)
    f = vnm.vnm_residual_norm(**t, **kw, want_stats=True)
    b = vnm.vnm_residual_norm_backward(**{**t, "h": f.h}, stats=f.stats, dx=cx, dh=ch, **kw)

    def loss(s):
        r = vnm.vnm_residual_norm(**s, **kw)
        return float((r.x.double() * cx).sum() + (r.h.double() * ch).sum())

    for name, grad in b._asdict().items():
        if grad is None:
            assert t[name] is None
            continue
        v = torch.randn(t[name].shape, generator=g).to(DEV)
        step = 2.0 ** -6
        diff = (loss({**t, name: t[name] + step * v}) - loss({**t, name: t[name] - step * v})) / (2 * step)
        terms = (grad.double() * v.double()).square().sum().sqrt()
        assert abs(diff - float((grad.double() * v.double()).sum())) <= 1e-2 * float(terms) + 1e-3, name


def test_backward_parts():
    """Outputs that are not asked for change nothing of the others; either gradient may be missing; in place of dh."""
    T, n = 33, 200
    t = on(make(T, n, "fp16", "fp16", "layer", "rms", -1))
    kw = dict(pre="layer", post="rms")
    f = vnm.vnm_residual_norm(**t, **kw, want_stats=True)
    t["h"] = f.h
    dx, dh = torch.randn(T, n, device=DEV).half(), torch.randn(T, n, device=DEV).half()
    full = vnm.vnm_residual_norm_backward(stats=f.stats, dx=dx, dh=dh, **t, **kw)
    b = vnm.vnm_residual_norm_backward(stats=f.stats, dx=dx, dh=dh, want_params=False, **t, **kw)
    assert torch.equal(b.h, full.h) and torch.equal(b.y, full.y) and b.gate is None and b.pre_weight is None
    b = vnm.vnm_residual_norm_backward(stats=f.stats, dx=dx, dh=dh, want_dh=False, want_dy=False, **t, **kw)
    assert b.h is None and b.y is None
    for name in ("gate", "post_weight", "pre_weight", "pre_bias"):
        assert torch.equal(getattr(b, name), getattr(full, name)), name
    zero = torch.zeros_like(dh)
    for part in (dict(dx=dx), dict(dh=dh)):
        a = vnm.vnm_residual_norm_backward(stats=f.stats, **part, **t, **kw)
        b = vnm.vnm_residual_norm_backward(stats=f.stats, dx=part.get("dx", zero), dh=part.get("dh", zero), **t, **kw)
        for name in ("h", "y", "gate", "post_weight"):
            assert torch.equal(getattr(a, name), getattr(b, name)), name
    again = vnm.vnm_residual_norm_backward(stats=f.stats, dx=dx, dh=dh, **t, **kw)
    assert all(x is None or torch.equal(x, y) for x, y in zip(again, full))


def test_backward_no_tokens():
    n = 64
    w = torch.ones(n, device=DEV)
    b = vnm.vnm_residual_norm_backward(torch.empty(0, n, device=DEV), torch.empty(0, 4, device=DEV), dx=torch.empty(0, n, device=DEV), pre="rms", pre_weight=w)
    assert b.h.shape == (0, n) and bool((b.pre_weight == 0).all())


def test_backward_on_streams_and_in_a_graph():
    T, n = 257, 768
    t = on(make(T, n, "fp32", "bf16", "layer", "rms", 50))
    kw = dict(pre="layer", post="rms", gate_tokens=50)
    f = vnm.vnm_residual_norm(**t, **kw, want_stats=True)
    s = {**t, "h": f.h}
    dx, dh = torch.randn(T, n, device=DEV).bfloat16(), torch.randn(T, n, device=DEV)
    call = lambda: vnm.vnm_residual_norm_backward(stats=f.stats, dx=dx, dh=dh, **s, **kw)
    want = call()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for k in range(6):
        with torch.cuda.stream(streams[k % 2]):
            got.append(call())
    torch.cuda.synchronize()
    for g in got:
        assert all(a is None or torch.equal(a, b) for a, b in zip(g, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fwd = vnm.vnm_residual_norm(**t, **kw, want_stats=True)
        out = vnm.vnm_residual_norm_backward(stats=fwd.stats, dx=dx, dh=dh, **{**t, "h": fwd.h}, **kw)
    for k in range(4):
        dx.copy_(torch.randn(T, n, device=DEV).bfloat16())
        graph.replay()
        eager = call()
        torch.cuda.synchronize()
        assert all(a is None or torch.equal(a, b) for a, b in zip(out, eager))
