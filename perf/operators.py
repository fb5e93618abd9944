"""8-bit sparse layers and the norms around them: cases that can be timed and compared.

Four operators that a Transformer block of V:N:M-sparse layers runs in 8 bits:
  quantize   int8 activations with one scale per token
  product    V:N:M-sparse product of int8 activations and int8 weights, one scale per token and per output channel
  norm       what stands between two blocks: the norm after a block, its gate, the residual scale, and the norm in front of
             the next block, whose result leaves in 16 bits, or as int8 activations that a product then reads
  backward   the gradients of that

With `own` false every operator is computed in its plain form with elementary torch operations, with `own` true by the
calls of this repository's package.  `listed()` gives the standing cases, `draw(rng)` one more of the same ranges, `prepare`
what a program holds before the call, `run` one pass, `work` the bytes and operations it cannot do without, `exact` its
outputs in 64 bits.
"""

import math

import torch

own = False
DEV = "cuda:0"
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def _quantize(name, T, n, x):
    return {"name": name, "op": "quantize", "T": T, "n": n, "x": x}


def _product(name, T, out, inn, V, M, y="fp16", bias=False):
    return {"name": name, "op": "product", "T": T, "out": out, "in": inn, "V": V, "M": M, "y": y, "bias": bias}


def _norm(name, T, n, h, x, pre, post="none", y=True, gate=0, scale=1.0, out=0, V=64, M=5):
    """gate: 0 none, -1 one row for all tokens, else the tokens that share a row.  out: width of the int8 layer that reads the
    norm's int8 result, 0 for a result of type `x`."""
    return {"name": name, "op": "norm", "T": T, "n": n, "h": h, "x": x, "pre": pre, "post": post, "y": y, "gate": gate,
            "scale": scale, "out": out, "V": V, "M": M}


def _backward(name, T, n, h, x, pre, post="none", gate=0, scale=1.0):
    return {"name": name, "op": "backward", "T": T, "n": n, "h": h, "x": x, "pre": pre, "post": post, "y": True,
            "gate": gate, "scale": scale}


def listed():
    return [
        # a batch of 24 sequences being decoded, in front of the down projection
        _quantize("quantize_t24_11008", 24, 11008, "fp16"),
        # a prompt of 4096 tokens in front of the q, k and v projections
        _quantize("quantize_t4096_4096", 4096, 4096, "bf16"),
        # decoding one sequence: the o projection, bound by latency and by the bytes of the weight
        _product("product_t1_4096x4096", 1, 4096, 4096, 64, 5),
        # decoding a batch of 16 with a sparser gate projection
        _product("product_t16_11008x4096", 16, 11008, 4096, 64, 8),
        # 8 images of 197 tokens through an encoder's qkv layer with its bias
        _product("product_t1576_2304x768", 1576, 2304, 768, 128, 8, bias=True),
        # a prompt of a length that is no multiple of any tile, 32-row blocks, bf16 result
        _product("product_t700_4096x4096", 700, 4096, 4096, 32, 6, y="bf16"),
        # prefill: the down projection of 4096 tokens
        _product("product_t4096_4096x11008", 4096, 4096, 11008, 64, 5),
        # decoding one sequence: residual addition and the norm in front of the next block
        _norm("norm_t1_4096", 1, 4096, "fp16", "fp16", "rms"),
        # 64 images of 197 tokens: the block's output scaled by channel, then the next block's norm
        _norm("norm_t12608_768", 12608, 768, "fp16", "fp16", "layer", gate=-1),
        # norms on both sides of the block, fp32 residual stream, int8 activations into the next layer
        _norm("norm_product_t2048_4096", 2048, 4096, "fp32", "bf16", "rms", post="rms", scale=0.5, out=4096),
        # training on 4096 tokens: gradients through the norms on both sides
        _backward("backward_t4096_4096", 4096, 4096, "bf16", "bf16", "rms", post="rms"),
        # training an encoder on 8 images with a gate per image and an fp32 residual stream
        _backward("backward_t1576_384", 1576, 384, "fp32", "fp16", "layer", gate=197),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi, odd):
    """A width: a multiple of 8 as a rule, any number with probability `odd`."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < odd else max(8, (n + 4) // 8 * 8)


def draw(rng):
    op = rng.choice(["quantize", "product", "product", "product", "norm", "norm", "backward"])
    if op == "quantize":
        n = _width(rng, 64, 11008, 0.3)
        return _drawn(_quantize("", _log_int(rng, 1, min(16384, (1 << 24) // n)), n, rng.choice(["fp16", "bf16", "fp32"])))
    if op == "product":
        out, inn = _width(rng, 96, 11008, 0.2), _width(rng, 96, 11008, 0.2)
        T = _log_int(rng, 1, int(min(12608, 1.5e11 / (out * inn))))
        return _drawn(_product("", T, out, inn, rng.choice([32, 64, 64, 128]), rng.choice([4, 5, 5, 6, 7, 8, 8, 10, 12, 16]),
                               y=rng.choice(["fp16", "fp16", "bf16", "fp32"]), bias=rng.random() < 0.4))
    n = _width(rng, 64, 8192, 0.2)
    T = _log_int(rng, 1, min(16384, (1 << 24) // n))
    x = rng.choice(["fp16", "bf16"])
    h = rng.choice([x, x, "fp32"])
    pre, post = rng.choice(["rms", "layer"]), rng.choice(["none", "none", "rms", "layer"])
    gate = rng.choice([0, 0, -1, rng.choice([64, 197, 577])])
    scale = rng.choice([1.0, 1.0, 0.5, 0.7071])
    if op == "backward":
        return _drawn(_backward("", T, n, h, x, pre, post, gate, scale))
    out = rng.choice([0, 0, 0, _width(rng, 96, 4096, 0.2)])
    return _drawn(_norm("", T, n, h, x, pre, post, True, gate, scale, out, rng.choice([32, 64, 128]), rng.choice([4, 5, 8])))


def _drawn(case):
    del case["name"]
    return case


# --- inputs ---------------------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)


def _activations(g, T, n):
    """N(0, 1) with one channel in a hundred ten times as large."""
    x = _randn(g, T, n)
    return x * torch.where(torch.rand(n, generator=g, device=DEV) < 0.01, 10.0, 1.0)


def _tokens_int8(x):
    """int8 values and one scale per row: scale = max |x| / 127, q = x * (127 / max |x|) rounded to the nearest, ties to even.
    The product is exact in 64 bits, so that a value next to a border falls on the right side."""
    top = x.abs().amax(1)
    scale = top / 127.0
    q = torch.round(x.double() * torch.where(top > 0, 127.0 / top, 0.0).double()[:, None])
    return q.to(torch.int8), scale


def _weight(g, out, inn, V, M):
    """An int8 V:N:M weight with a scale per output channel: the triple of its storage form, and dense in fp32."""
    R, B = -(-out // V), -(-inn // M)
    real = torch.arange(B * M, device=DEV).view(1, B, M) < inn      # columns past the last one are kept last, with value 0
    key = torch.rand(R, B, M, generator=g, device=DEV) + torch.where(real, 0.0, 2.0)
    col = key.argsort(2)[:, :, :4].sort(2).values                    # the 4 kept columns of every block
    first = torch.tensor([0, 0, 0, 1, 1, 2], device=DEV)
    second = torch.tensor([1, 2, 3, 2, 3, 3], device=DEV)
    pair = torch.randint(0, 6, (R * V, B), generator=g, device=DEV)  # which two of them a row keeps
    pos = torch.stack([first[pair], second[pair]], 2)                # [out_pad, B, 2]
    kept = torch.gather(col.repeat_interleave(V, 0), 2, pos) + torch.arange(B, device=DEV)[None, :, None] * M
    value = _randn(g, R * V, B, 2) * 0.02
    value = torch.where((kept < inn) & (torch.arange(R * V, device=DEV) < out)[:, None, None], value, 0.0)
    q, scale = _tokens_int8(value.view(R * V, 2 * B))
    dense = torch.zeros(R * V, B * M, device=DEV)
    dense.scatter_(1, kept.view(R * V, 2 * B), q.float())
    nibble = (pos[:, :, 0] | pos[:, :, 1] << 2).to(torch.uint8)
    if B % 2:
        nibble = torch.cat([nibble, torch.full_like(nibble[:, :1], 4)], 1)
    return {"values": q.reshape(-1), "meta": (nibble[:, 0::2] | nibble[:, 1::2] << 4).reshape(-1),
            "colidx": col.to(torch.uint8).reshape(-1), "scale": scale[:out].contiguous(),
            "dense": dense[:out, :inn].contiguous()}


def _layer(g, case, inn):
    """The int8 layer of a case: its weight and, for the framework's call, the handle that a program keeps for it."""
    w = _weight(g, case["out"], inn, case["V"], case["M"])
    w["bias"] = (_randn(g, case["out"]) * 0.1).half() if case.get("bias") else None
    if own:
        import paper_2410_16135_amd as vnm
        w["handle"] = vnm.vnm_pack_i8(vnm.CompressedI8(w["values"], w["meta"], w["colidx"], None, w["scale"], case["out"],
                                                       inn, case["V"], case["M"]))
    return w


def _normed(v, kind, weight, bias, eps):
    """(result, mean, reciprocal deviation) of a norm over the rows of v, in v's own precision."""
    if kind == "none":
        return v, torch.zeros_like(v[:, :1]), torch.ones_like(v[:, :1])
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    r = 1.0 / torch.sqrt((v - mean).square().mean(1, keepdim=True) + eps)
    x = (v - mean) * r * weight
    return x + bias if bias is not None else x, mean, r


def prepare(case, seed):
    g = _generator(seed)
    T = case["T"]
    if case["op"] == "quantize":
        return {"case": case, "x": _activations(g, T, case["n"]).to(TYPES[case["x"]])}
    if case["op"] == "product":
        inn = case["in"]
        q, scale = _tokens_int8(_activations(g, T, inn).half().float())
        rows = torch.zeros(T, -(-inn // 16) * 16, dtype=torch.int8, device=DEV)   # rows 16-byte aligned, as the quantizer leaves them
        rows[:, :inn] = q
        return {"case": case, "q": rows[:, :inn], "scale": scale, "w": _layer(g, case, inn)}
    n, xt, ht = case["n"], TYPES[case["x"]], TYPES[case["h"]]
    s = {"case": case, "h": _activations(g, T, n).to(ht), "y": _randn(g, T, n).to(xt)}
    for which in ("pre", "post"):
        kind = case[which]
        s[which + "_weight"] = (1.0 + 0.1 * _randn(g, n)).to(xt) if kind != "none" else None
        s[which + "_bias"] = (0.1 * _randn(g, n)).to(xt) if kind == "layer" else None
    rows = 0 if case["gate"] == 0 else 1 if case["gate"] < 0 else -(-T // case["gate"])
    s["gate"] = (0.5 + 0.2 * _randn(g, rows, n)).to(xt) if rows else None
    s["eps"] = 1e-5
    if case["op"] == "norm":
        if case["out"]:
            s["w"] = _layer(g, case, n)
        return s
    # what the forward pass left: the new residual stream, and mean and reciprocal deviation of both norms
    y, ym, yr = _normed(s["y"].float(), case["post"], *_weights(s, "post", torch.float32))
    h = case["scale"] * s["h"].float() + _gate(s, torch.float32, y)
    _, hm, hr = _normed(h, case["pre"], *_weights(s, "pre", torch.float32))
    s["h"], s["stats"] = h.to(ht), torch.cat([ym, yr, hm, hr], 1)
    s["dx"], s["dh"] = _randn(g, T, n).to(xt), _randn(g, T, n).to(ht)
    return s


def _weights(s, which, dtype):
    w, b = s[which + "_weight"], s[which + "_bias"]
    return (None if w is None else w.to(dtype)), (None if b is None else b.to(dtype)), s["eps"]


def _gate_rows(s, dtype):
    gate, tokens = s["gate"].to(dtype), s["case"]["gate"]
    return gate if tokens < 0 else gate.repeat_interleave(tokens, 0)[: s["case"]["T"]]


def _gate(s, dtype, y):
    return y if s["gate"] is None else _gate_rows(s, dtype) * y


# --- one pass -------------------------------------------------------------------------------------------------------

def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    if case["op"] == "quantize":
        q, scale = _tokens_int8(state["x"].float())
        return {"q": q, "scale": scale}
    if case["op"] == "product":
        return _plain_product(state["q"], state["scale"], state["w"], TYPES[case["y"]])
    if case["op"] == "norm":
        y, _, _ = _normed(state["y"].float(), case["post"], *_weights(state, "post", torch.float32))
        h = case["scale"] * state["h"].float() + _gate(state, torch.float32, y)
        x, _, _ = _normed(h, case["pre"], *_weights(state, "pre", torch.float32))
        if not case["out"]:
            return {"h": h.to(state["h"].dtype), "x": x.to(state["y"].dtype)}
        return {"h": h.to(state["h"].dtype), "y": _plain_product(*_tokens_int8(x), state["w"], state["y"].dtype)}
    return _plain_backward(state)


def _plain_product(q, scale, w, dtype):
    y = torch.matmul(q.float(), w["dense"].t()) * w["scale"] * scale[:, None]
    if w["bias"] is not None:
        y = y + w["bias"].float()
    return y.to(dtype)


def _plain_backward(s):
    case, f = s["case"], torch.float32
    ym, yr, hm, hr = s["stats"].unbind(1)
    hhat = (s["h"].float() - hm[:, None]) * hr[:, None]
    dx = s["dx"].float()
    got = {"pre_weight": (dx * hhat).sum(0)}
    if s["pre_bias"] is not None:
        got["pre_bias"] = dx.sum(0)
    d = s["dh"].float() + _through_norm(dx * s["pre_weight"].float(), hhat, hr, case["pre"])
    got["dh"] = (case["scale"] * d).to(s["h"].dtype)
    yhat = (s["y"].float() - ym[:, None]) * yr[:, None]
    p = yhat
    if s["post_weight"] is not None:
        p = p * s["post_weight"].float()
    if s["post_bias"] is not None:
        p = p + s["post_bias"].float()
    if s["gate"] is not None:
        got["gate"] = _group_sums(d * p, case["gate"])
        d = d * _gate_rows(s, f)
    if case["post"] != "none":
        got["post_weight"] = (d * yhat).sum(0)
        if s["post_bias"] is not None:
            got["post_bias"] = d.sum(0)
        d = _through_norm(d * s["post_weight"].float(), yhat, yr, case["post"])
    got["dy"] = d.to(s["y"].dtype)
    return got


def _through_norm(g, xhat, r, kind):
    """Gradient of a norm's input, from the gradient g of the normalised values."""
    d = g - xhat * (g * xhat).mean(1, keepdim=True)
    if kind == "layer":
        d = d - g.mean(1, keepdim=True)
    return d * r[:, None]


def _group_sums(v, tokens):
    """Sums over the tokens that share a gate row."""
    T, n = v.shape
    if tokens < 0:
        return v.sum(0, keepdim=True)
    rows = -(-T // tokens)
    padded = torch.zeros(rows * tokens, n, dtype=v.dtype, device=v.device)
    padded[:T] = v
    return padded.view(rows, tokens, n).sum(1)


def _norm_arguments(s):
    case = s["case"]
    return dict(gate=None if s["gate"] is None else s["gate"][0] if case["gate"] < 0 else s["gate"],
                gate_tokens=max(0, case["gate"]), residual_scale=case["scale"], post=case["post"], pre=case["pre"],
                post_weight=s["post_weight"], post_bias=s["post_bias"], pre_weight=s["pre_weight"], pre_bias=s["pre_bias"])


def _run_own(s):
    import paper_2410_16135_amd as vnm
    case = s["case"]
    if case["op"] == "quantize":
        q, scale = vnm.vnm_quantize_x(s["x"])
        return {"q": q, "scale": scale}
    if case["op"] == "product":
        return vnm.vnm_spmm_i8(s["q"], s["scale"], s["w"]["handle"], bias=s["w"]["bias"], out_dtype=TYPES[case["y"]])
    if case["op"] == "norm":
        r = vnm.vnm_residual_norm(s["h"], s["y"], post_eps=s["eps"], pre_eps=s["eps"], int8=bool(case["out"]),
                                  **_norm_arguments(s))
        if not case["out"]:
            return {"h": r.h, "x": r.x}
        return {"h": r.h, "y": vnm.vnm_spmm_i8(r.x, r.scale, s["w"]["handle"], out_dtype=s["y"].dtype)}
    d = vnm.vnm_residual_norm_backward(s["h"], s["stats"], dx=s["dx"], dh=s["dh"], y=s["y"], **_norm_arguments(s))
    got = {"dh": d.h, "dy": d.y, "pre_weight": d.pre_weight}
    if s["pre_bias"] is not None:
        got["pre_bias"] = d.pre_bias
    if s["gate"] is not None:
        got["gate"] = d.gate.view(-1, case["n"])
    if case["post"] != "none":
        got["post_weight"] = d.post_weight
        if s["post_bias"] is not None:
            got["post_bias"] = d.post_bias
    return got


# --- what a pass cannot do without ----------------------------------------------------------------------------------

def _product_work(T, out, inn, V, M, y_bytes, bias):
    """The kept weights (int8, two 2-bit positions, four column numbers per block), activations, scales and result; a
    multiplication and an addition per kept weight and token."""
    R, B = -(-out // V), -(-inn // M)
    weight = out * 2 * B + out * B / 2 + 4 * R * B + 4 * out + (2 * out if bias else 0)
    return weight, T * inn + 4 * T, T * out * y_bytes, 2.0 * T * out * 2 * B


def work(case):
    size = {"fp16": 2, "bf16": 2, "fp32": 4}
    T = case["T"]
    if case["op"] == "quantize":
        n = case["n"]
        return {"bytes": T * n * (size[case["x"]] + 1) + 4 * T, "flops": 2 * T * n}
    if case["op"] == "product":
        w, x, y, flops = _product_work(T, case["out"], case["in"], case["V"], case["M"], size[case["y"]], case["bias"])
        return {"bytes": w + x + y, "flops": flops}
    n, hb, xb = case["n"], size[case["h"]], size[case["x"]]
    gate = 0 if case["gate"] == 0 else 1 if case["gate"] < 0 else -(-T // case["gate"])
    params = {"none": 0, "rms": 1, "layer": 2}
    vectors = n * (params[case["pre"]] + params[case["post"]] + gate)
    if case["op"] == "norm":
        b = T * n * (2 * hb + xb) + vectors * xb                   # residual stream in and out, the block's output
        if not case["out"]:
            return {"bytes": b + T * n * xb, "flops": 12 * T * n}
        w, _, y, flops = _product_work(T, case["out"], n, case["V"], case["M"], xb, False)
        return {"bytes": b + w + y, "flops": 12 * T * n + flops}   # (the int8 activations need not leave the chip)
    # dx, dh, h and y in (y only where a norm or a gate needs it), the gradients of h and y out
    need_y = case["post"] != "none" or gate
    return {"bytes": T * n * (3 * hb + (2 + bool(need_y)) * xb) + 16 * T + vectors * (xb + 4), "flops": 24 * T * n}


# --- the definition in 64 bits --------------------------------------------------------------------------------------

def _exact_norm(v, kind, w, b, eps):
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.sum(1, keepdim=True) / v.shape[1]
    out = v * torch.rsqrt((v * v).sum(1, keepdim=True) / v.shape[1] + eps) * w.double()
    return out if b is None else out + b.double()


def _exact_product(q, scale, w, bias):
    y = (q.double() @ w["dense"].double().t()) * (scale.double()[:, None] * w["scale"].double()[None, :])
    return y if bias is None else y + bias.double()


def _exact_norm_input_gradient(g, xhat, r, kind):
    n = g.shape[1]
    d = n * g - xhat * (g * xhat).sum(1, keepdim=True)
    if kind == "layer":
        d -= g.sum(1, keepdim=True)
    return d * (r / n)


def exact(case, seed):
    s = prepare(case, seed)
    T = case["T"]
    if case["op"] == "quantize":
        x = s["x"].double()
        top = x.abs().max(1).values
        inverse = torch.where(top > 0, 127.0 / top, 0.0).float().double()      # the factor itself is an fp32 number
        return {"q": torch.round(x * inverse[:, None]).to(torch.int8), "scale": top / 127.0}
    if case["op"] == "product":
        return _exact_product(s["q"], s["scale"], s["w"], s["w"]["bias"])
    row = None if s["gate"] is None else torch.zeros(T, dtype=torch.long, device=DEV) if case["gate"] < 0 \
        else torch.arange(T, device=DEV) // case["gate"]
    gate = 1.0 if row is None else s["gate"].double()[row]
    y = s["y"].double()
    if case["op"] == "norm":
        h = s["h"].double() * case["scale"] + gate * _exact_norm(y, case["post"], s["post_weight"], s["post_bias"], s["eps"])
        x = _exact_norm(h, case["pre"], s["pre_weight"], s["pre_bias"], s["eps"])
        if not case["out"]:
            return {"h": h, "x": x}
        top = x.abs().max(1).values
        q = torch.round(x * (127.0 / top)[:, None])
        return {"h": h, "y": _exact_product(q, top / 127.0, s["w"], None)}
    stats = s["stats"].double()
    hhat, yhat = (s["h"].double() - stats[:, 2:3]) * stats[:, 3:4], (y - stats[:, 0:1]) * stats[:, 1:2]
    dx = s["dx"].double()
    d = s["dh"].double() + _exact_norm_input_gradient(dx * s["pre_weight"].double(), hhat, stats[:, 3:4], case["pre"])
    got = {"dh": d * case["scale"], "pre_weight": torch.einsum("tn,tn->n", dx, hhat)}
    if s["pre_bias"] is not None:
        got["pre_bias"] = dx.sum(0)
    if row is not None:
        p = yhat if s["post_weight"] is None else yhat * s["post_weight"].double()
        p = p if s["post_bias"] is None else p + s["post_bias"].double()
        got["gate"] = torch.zeros(s["gate"].shape, dtype=torch.float64, device=DEV).index_add_(0, row, d * p)
    dz = d * gate
    if case["post"] != "none":
        got["post_weight"] = torch.einsum("tn,tn->n", dz, yhat)
        if s["post_bias"] is not None:
            got["post_bias"] = dz.sum(0)
        dz = _exact_norm_input_gradient(dz * s["post_weight"].double(), yhat, stats[:, 1:2], case["post"])
    got["dy"] = dz
    return got
