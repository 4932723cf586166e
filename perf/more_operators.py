"""Rows that are normalised, laid down in 8 or 4 bits with block scales, and multiplied in that form, as cases that can be timed and
compared: the plain forms in torch, or, with `own` set, the calls of the library's binding.

A case is one of seven kinds:

  norm        root-mean-square norm of x, or of x + residual, into the type of x or into 8 bits with scales
  backward    its gradients: of the rows, with what comes down the residual stream, and of the weight
  quantize    a matrix into blocks of 32 that share a scale, along its rows, its columns or both
  dequantize  such a matrix back into numbers
  product     C = A . B^T of two such matrices, with the fused epilogue of the other products
  layer       norm into 8 bits, and the product that reads it
  train       a linear layer's step: the operands quantised along both axes, its output and both gradients

A block of 32 elements shares a scale that is a power of two, 2^(floor(log2 of its largest magnitude) - emax), held as the power plus
127 in 8 bits; its elements are x / scale, rounded to nearest even into the format and cut to its largest value.  Rows are filled up to
whole blocks with zeros; the scales of a block of columns lie side by side, [block][row].  4-bit values are compared as the numbers
that they stand for, which the operator next to them gives back.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
# bits of the mantissa, lowest and highest power of two, largest value, bytes of a block of 32
FORMATS = {"e4m3": (3, -6, 8, 448.0, 32), "e5m2": (2, -14, 15, 57344.0, 32), "e2m1": (1, 0, 2, 6.0, 16)}
FLOAT8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
EPS = 1e-5


def _norm(name, dtype, rows, cols, residual=True, out="plain", offset=0.0):
    return dict(name=name, kind="norm", dtype=dtype, rows=rows, cols=cols, residual=residual, out=out, offset=offset)


def _backward(name, dtype, rows, cols, stream=True, offset=0.0):
    return dict(name=name, kind="backward", dtype=dtype, rows=rows, cols=cols, stream=stream, offset=offset)


def _quantize(name, dtype, rows, cols, fmt, axes):
    return dict(name=name, kind="quantize", dtype=dtype, rows=rows, cols=cols, format=fmt, axes=axes)


def _product(name, a, b, out, m, n, k, bias=False, relu=False, residual=False):
    return dict(name=name, kind="product", a=a, b=b, out=out, m=m, n=n, k=k, bias=bias, relu=relu, residual=residual)


def listed():
    return [
        # the residual stream of one decoding step of 4 sequences: latency
        _norm("norm_decode", "bf16", 4, 4096),
        # the same of a long prompt, into the operand of the next product: memory
        _norm("norm_prompt_8bit", "bf16", 16384, 8192, out="e4m3"),
        # the gradients of a training step of 8192 tokens
        _backward("norm_backward", "bf16", 8192, 5120),
        # the same in fp32, at odd sizes, for weights kept as distances from one
        _backward("norm_backward_f32", "f32", 1021, 2039, stream=False, offset=1.0),
        # a layer's weights into 4 bits, and what they then stand for
        _quantize("quantize_weights_4bit", "bf16", 16384, 4096, "e2m1", "rows"),
        # a ragged batch's gradients into 8 bits along both axes, for the two products that read them
        _quantize("quantize_gradients_both", "f16", 4099, 1003, "e5m2", "both"),
        # 4-bit weights for an operator that takes bf16
        dict(name="dequantize_weights_4bit", kind="dequantize", dtype="bf16", rows=16384, cols=4096, format="e2m1"),
        # one decoding step of 4 sequences against 4-bit weights: memory, latency
        _product("product_decode", "e4m3", "e2m1", "bf16", 4, 8192, 4096, residual=True),
        # a long prompt in 4 bits: the matrix cores
        _product("product_prompt_4bit", "e2m1", "e2m1", "bf16", 8192, 8192, 8192),
        # odd sizes, with bias and activation
        _product("product_odd", "e4m3", "e4m3", "f16", 2039, 1021, 1000, bias=True, relu=True),
        # norm and product of a chunk of a prompt
        dict(name="layer_chunk", kind="layer", dtype="bf16", format="e4m3", b="e2m1", m=333, n=5120, k=4096),
        # a linear layer's training step, gradients in the format of the wider range
        dict(name="train_step", kind="train", dtype="bf16", format="e4m3", gradients="e5m2", m=4096, n=4096, k=4096),
    ]


def _log(rng, low, high):
    """A whole number between `low` and `high`, spread over its logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    kind = rng.choice(("norm", "norm", "backward", "quantize", "quantize", "dequantize", "product", "product", "product", "layer", "train"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    fmt = rng.choice(("e4m3", "e5m2", "e2m1"))
    if kind in ("norm", "backward", "quantize", "dequantize"):
        cols = _log(rng, 32, 16384)
        if rng.random() < 0.5:
            cols = max(32, cols // 64 * 64)
        rows = _log(rng, 1, max(2, min(65536, 30000000 // cols)))
        if kind == "norm":
            return dict(kind=kind, dtype=dtype, rows=rows, cols=cols, residual=rng.random() < 0.6,
                        out=rng.choice(("plain", "e4m3", "e5m2")), offset=rng.choice((0.0, 1.0)))
        if kind == "backward":
            return dict(kind=kind, dtype=dtype, rows=rows, cols=cols, stream=rng.random() < 0.6, offset=rng.choice((0.0, 1.0)))
        if kind == "quantize":
            return dict(kind=kind, dtype=dtype, rows=rows, cols=cols, format=fmt, axes=rng.choice(("rows", "columns", "both")))
        return dict(kind=kind, dtype=dtype, rows=rows, cols=cols, format=fmt)
    n, k = _log(rng, 64, 8192), _log(rng, 64, 8192)
    if rng.random() < 0.6:
        n, k = max(64, n // 64 * 64), max(64, k // 64 * 64)
    m = _log(rng, 1, 4096)
    if kind == "layer":
        return dict(kind=kind, dtype=rng.choice(("bf16", "f16")), format=rng.choice(("e4m3", "e5m2")), b=fmt, m=m, n=n, k=k)
    if kind == "train":
        return dict(kind=kind, dtype=rng.choice(("bf16", "f16")), format=rng.choice(("e4m3", "e2m1")),
                    gradients=rng.choice(("e4m3", "e5m2")), m=max(m, 32), n=min(n, 4096), k=min(k, 4096))
    a = rng.choice(("e4m3", "e4m3", "e5m2", "e2m1"))
    return dict(kind=kind, a=a, b=fmt, out=rng.choice(("bf16", "f16", "f32") if a == fmt == "e2m1" else ("bf16", "f16")), m=m, n=n, k=k,
                bias=rng.random() < 0.4, relu=rng.random() < 0.3, residual=rng.random() < 0.4)


def _blocks(n):
    return (n + 31) // 32


# ---- the plain forms ------------------------------------------------------------------------------------------------

def _power(e):
    """2^e of whole numbers from -126 to 127, exactly."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _rounded(q, fmt):
    """q (float32) to nearest even in the format, cut to its largest value."""
    bits, low, _, top, _ = FORMATS[fmt]
    step = (torch.frexp(q)[1] - 1).clamp(min=low) - bits
    return (torch.round(q * _power(-step)) * _power(step)).clamp(-top, top)


def _quantized(x, fmt):
    """x [rows][cols] float32 -> (values float32 [rows][whole blocks], scales as whole numbers [blocks][rows])."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, -cols % 32)).unflatten(1, (-1, 32))
    top = x.abs().amax(2)
    e = (torch.frexp(top)[1] - 1 - FORMATS[fmt][2]).clamp(min=-127)
    e = torch.where(top == 0, torch.full_like(e, -127), e)
    values = _rounded(x * _power(-e)[..., None], fmt)
    return values.flatten(1), (e + 127).t().contiguous()


def _numbers(values, scales):
    """What values and scales stand for."""
    e = scales.t().to(torch.int32) - 127
    whole = _power(e.clamp(min=-126)) * torch.where(e < -126, 0.5, 1.0)
    return (values.unflatten(1, (-1, 32)) * whole[..., None]).flatten(1)


def _codes(values, fmt):
    """Values in their format, packed as they lie in memory."""
    if fmt in FLOAT8:
        return values.to(FLOAT8[fmt]).view(torch.uint8)
    table = torch.zeros(13, dtype=torch.uint8, device=values.device)
    table[torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], device=values.device)] = torch.arange(8, dtype=torch.uint8, device=values.device)
    code = table[(values.abs() * 2).long()] | (torch.signbit(values).to(torch.uint8) << 3)
    return (code[:, 0::2] | (code[:, 1::2] << 4)).contiguous()


def _decoded(codes, fmt):
    if fmt in FLOAT8:
        return codes.view(FLOAT8[fmt]).float()
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=codes.device)
    return torch.stack((table[(codes & 15).long()], table[(codes >> 4).long()]), 2).flatten(1)


def _shown(values, scales, fmt):
    """Outputs in 8 bits: the values that they stand for, in a type of 8 bits."""
    return values.to(FLOAT8[fmt]), scales.to(torch.uint8).view(torch.float8_e8m0fnu)


def _plain_norm(s, case):
    h = s["x"].float()
    if "residual" in s:
        h = (h + s["residual"].float()).to(s["x"].dtype).float()  # (the stream is kept in the type of x)
    rstd = (h.double().square().mean(1, keepdim=True) + EPS).rsqrt().float()
    return h, h * rstd * (s["weight"].float() + case.get("offset", 0.0)), rstd


def _plain_backward(s, case):
    h, grad = s["h"].float(), s["grad"].float()
    xhat = h * s["rstd"][:, None]
    g = grad * (s["weight"].float() + case["offset"])
    grad_x = s["rstd"][:, None] * (g - xhat * (g * xhat).mean(1, keepdim=True))
    if "stream" in s:
        grad_x = grad_x + s["stream"].float()
    return grad_x.to(s["h"].dtype), (grad * xhat).sum(0).to(s["weight"].dtype)


def _plain_run(s, case):
    kind = case["kind"]
    if kind in ("norm", "layer"):
        h, y, rstd = _plain_norm(s, case)
        stream = h.to(s["x"].dtype) if "residual" in s else None
        if kind == "layer":
            c = _numbers(*_quantized(y, case["format"])) @ _numbers(_decoded(s["b"][0], case["b"]), s["b"][1]).t()
            return dict(stream=stream, c=c.to(s["x"].dtype))
        if case["out"] == "plain":
            return dict(stream=stream, y=y.to(s["x"].dtype), rstd=rstd[:, 0])
        values, scales = _shown(*_quantized(y, case["out"]), case["out"])
        return dict(stream=stream, values=values, scales=scales)
    if kind == "backward":
        return _plain_backward(s, case)
    if kind == "quantize":
        found = {}
        x = s["x"].float()
        for axis, m in (("rows", x), ("columns", x.t())):
            if case["axes"] in (axis, "both"):
                values, scales = _quantized(m, case["format"])
                if case["format"] in FLOAT8:
                    found[axis], found[axis + "_scales"] = _shown(values, scales, case["format"])
                else:
                    found[axis] = _numbers(values, scales)[:, :m.shape[1]].to(s["x"].dtype)
                    found[axis + "_scales"] = scales.to(torch.uint8).view(torch.float8_e8m0fnu)
        return found
    if kind == "dequantize":
        return _numbers(_decoded(s["a"][0], case["format"]), s["a"][1])[:, :case["cols"]].to(DTYPES[case["dtype"]])
    if kind == "train":
        x, w, g = s["x"].float(), s["w"].float(), s["grad"].float()
        f, e = case["format"], case["gradients"]
        y = _numbers(*_quantized(x, f)) @ _numbers(*_quantized(w, f)).t()
        grad_x = _numbers(*_quantized(g, e)) @ _numbers(*_quantized(w.t(), f)).t()
        grad_w = _numbers(*_quantized(g.t(), e)) @ _numbers(*_quantized(x.t(), f)).t()
        return dict(y=y.to(s["x"].dtype), grad_x=grad_x.to(s["x"].dtype), grad_w=grad_w.to(s["x"].dtype))
    c = _numbers(_decoded(s["a"][0], case["a"]), s["a"][1]) @ _numbers(_decoded(s["b"][0], case["b"]), s["b"][1]).t()
    if "bias" in s:
        c = c + s["bias"].float()
    if "residual" in s:
        c = c + s["residual"].float()
    if case["relu"]:
        c = c.clamp(min=0.0)
    return c.to(DTYPES[case["out"]])


# ---- what a program has before a call -------------------------------------------------------------------------------

def _inputs(case, seed):
    device = torch.device("cuda")
    g = torch.Generator(device=device).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=device, dtype=torch.float32)

    def activations(rows, cols):
        """Rows of unlike size, with a few columns that are much larger than the others."""
        wide = torch.where(torch.rand(cols, generator=g, device=device) < 0.01, 20.0, 1.0)
        return normal(rows, cols) * wide * torch.exp(0.5 * normal(rows, 1))

    def matrix(rows, cols, fmt, size):
        values, scales = _quantized(normal(rows, cols) * size, fmt)
        return _codes(values, fmt), scales.to(torch.uint8)

    s, kind = dict(case=case), case["kind"]
    if kind in ("norm", "backward"):
        dtype = DTYPES[case["dtype"]]
        x = activations(case["rows"], case["cols"])
        s["weight"] = (0.2 * normal(case["cols"]) + 1.0 - case["offset"]).to(dtype)
        if kind == "norm":
            s["x"] = x.to(dtype)
            if case["residual"]:
                s["residual"] = activations(case["rows"], case["cols"]).to(dtype)
        else:
            s["h"] = x.to(dtype)
            s["rstd"] = (s["h"].double().square().mean(1) + EPS).rsqrt().float()
            s["grad"] = (0.01 * normal(case["rows"], case["cols"])).to(dtype)
            if case["stream"]:
                s["stream"] = (0.01 * normal(case["rows"], case["cols"])).to(dtype)
    elif kind == "quantize":
        s["x"] = activations(case["rows"], case["cols"]).to(DTYPES[case["dtype"]])
    elif kind == "dequantize":
        s["a"] = matrix(case["rows"], case["cols"], case["format"], 0.02)
    elif kind == "product":
        m, n, k, dtype = case["m"], case["n"], case["k"], DTYPES[case["out"]]
        s["a"], s["b"] = matrix(m, k, case["a"], 1.0), matrix(n, k, case["b"], k ** -0.5)
        if case["bias"]:
            s["bias"] = normal(n).to(dtype)
        if case["residual"]:
            s["residual"] = normal(m, n).to(dtype)
    elif kind == "layer":
        dtype = DTYPES[case["dtype"]]
        s["x"], s["residual"] = activations(case["m"], case["k"]).to(dtype), activations(case["m"], case["k"]).to(dtype)
        s["weight"] = (0.2 * normal(case["k"]) + 1.0).to(dtype)
        s["b"] = matrix(case["n"], case["k"], case["b"], case["k"] ** -0.5)
    else:
        dtype = DTYPES[case["dtype"]]
        s["x"] = activations(case["m"], case["k"]).to(dtype)
        s["w"] = (normal(case["n"], case["k"]) * case["k"] ** -0.5).to(dtype)
        s["grad"] = (0.01 * normal(case["m"], case["n"])).to(dtype)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    for name, rows in (("a", case.get("rows", case.get("m"))), ("b", case.get("n"))):
        if name in s:  # (the rows of scales are 4-byte words)
            codes, scales = s[name]
            room = torch.zeros(scales.shape[0], (rows + 3) // 4 * 4, dtype=torch.uint8, device=scales.device)
            room[:, :rows] = scales
            s[name] = codes, room[:, :rows]
    return s


def run(state):
    return _run_own(state, state["case"]) if own else _plain_run(state, state["case"])


# ---- the library's calls --------------------------------------------------------------------------------------------

def _room(s, name, make):
    """Memory of the program's own: made at the first pass, used again by the next."""
    if name not in s:
        s[name] = make()
    return s[name]


def _run_own(s, case):
    from paper_2210_09603_amd import binding as hb

    formats = dict(e4m3=hb.HIDET_MX_E4M3, e5m2=hb.HIDET_MX_E5M2, e2m1=hb.HIDET_MX_E2M1)
    kind, cuda = case["kind"], torch.device("cuda")

    def operand(name, fmt, rows, cols):
        return _room(s, name + "_mx", lambda: hb.make_mx(rows, cols, formats[fmt], values=s[name][0], scales=s[name][1]))

    def quantized(name, fmt, rows, cols):
        return _room(s, name, lambda: hb.make_mx(rows, cols, formats[fmt], device=cuda))

    def matrix(name, rows, cols, dtype):
        return _room(s, name, lambda: torch.empty((rows, cols), dtype=dtype, device=cuda))

    def product(name, a, b, m, n, k, dtype, epilogue=None):
        c = matrix(name, m, n, dtype)
        workspace = _room(s, name + "_workspace",
                          lambda: torch.empty(hb.hidet_mx_gemm_workspace_bytes(a, b), dtype=torch.uint8, device=cuda))
        hb.hidet_mx_gemm(a, b, c, epilogue=epilogue, workspace=workspace)
        return c

    def shown(q, fmt):
        values, scales = q.tensors
        return values.view(FLOAT8[fmt]) if fmt in FLOAT8 else None, scales.view(torch.float8_e8m0fnu)

    if kind in ("norm", "layer"):
        rows, cols = s["x"].shape
        stream = matrix("stream", rows, cols, s["x"].dtype) if "residual" in s else None
        if kind == "norm" and case["out"] == "plain":
            y, rstd = matrix("y", rows, cols, s["x"].dtype), _room(s, "rstd", lambda: torch.empty(rows, device=cuda))
            hb.hidet_rms_norm(s["x"], s["weight"], y=y, residual=s.get("residual"), sum=stream, rstd=rstd, eps=EPS, offset=case["offset"])
            return dict(stream=stream, y=y, rstd=rstd)
        fmt = case["out"] if kind == "norm" else case["format"]
        q = quantized("q", fmt, rows, cols)
        hb.hidet_rms_norm(s["x"], s["weight"], quantized=q, residual=s.get("residual"), sum=stream, eps=EPS, offset=case.get("offset", 0.0))
        if kind == "norm":
            values, scales = shown(q, fmt)
            return dict(stream=stream, values=values, scales=scales)
        return dict(stream=stream, c=product("c", q, operand("b", case["b"], case["n"], cols), rows, case["n"], cols, s["x"].dtype))
    if kind == "backward":
        rows, cols = s["h"].shape
        grad_x = matrix("grad_x", rows, cols, s["h"].dtype)
        grad_weight = _room(s, "grad_weight", lambda: torch.empty(cols, dtype=s["weight"].dtype, device=cuda))
        workspace = _room(s, "workspace", lambda: torch.empty(hb.hidet_rms_norm_backward_workspace_bytes(rows, cols), dtype=torch.uint8,
                                                              device=cuda))
        hb.hidet_rms_norm_backward(s["grad"], s["h"], s["rstd"], s["weight"], grad_x, grad_weight, workspace, grad_sum=s.get("stream"),
                                   offset=case["offset"])
        return grad_x, grad_weight
    if kind == "quantize":
        rows, cols = s["x"].shape
        by_rows = quantized("q_rows", case["format"], rows, cols) if case["axes"] != "columns" else None
        by_columns = quantized("q_columns", case["format"], cols, rows) if case["axes"] != "rows" else None
        hb.hidet_mx_quantize(s["x"], by_rows=by_rows, by_columns=by_columns)
        found = {}
        for axis, q, (r, c) in (("rows", by_rows, (rows, cols)), ("columns", by_columns, (cols, rows))):
            if q is not None:
                found[axis], found[axis + "_scales"] = shown(q, case["format"])
                if case["format"] not in FLOAT8:
                    found[axis] = matrix("y_" + axis, r, c, s["x"].dtype)
                    hb.hidet_mx_dequantize(q, found[axis])
        return found
    if kind == "dequantize":
        y = matrix("y", case["rows"], case["cols"], DTYPES[case["dtype"]])
        hb.hidet_mx_dequantize(operand("a", case["format"], case["rows"], case["cols"]), y)
        return y
    m, n, k = case["m"], case["n"], case["k"]
    if kind == "train":
        f, e, dtype = case["format"], case["gradients"], s["x"].dtype
        x, xt, w, wt = quantized("xq", f, m, k), quantized("xtq", f, k, m), quantized("wq", f, n, k), quantized("wtq", f, k, n)
        g, gt = quantized("gq", e, m, n), quantized("gtq", e, n, m)
        for t, by_rows, by_columns in ((s["x"], x, xt), (s["w"], w, wt), (s["grad"], g, gt)):
            hb.hidet_mx_quantize(t, by_rows=by_rows, by_columns=by_columns)
        return dict(y=product("y", x, w, m, n, k, dtype), grad_x=product("grad_x", g, wt, m, k, n, dtype),
                    grad_w=product("grad_w", gt, xt, n, k, m, dtype))
    epilogue = None
    if case["bias"] or case["relu"] or case["residual"]:
        epilogue = _room(s, "epilogue", lambda: hb.make_epilogue(bias=s.get("bias"), residual=s.get("residual"), relu=case["relu"],
                                                                 bias_axis=hb.HIDET_BIAS_PER_COL if case["bias"] else hb.HIDET_BIAS_NONE))
    return product("c", operand("a", case["a"], m, k), operand("b", case["b"], n, k), m, n, k, DTYPES[case["out"]], epilogue)


# ---- work, and the definitions in 64 bits -----------------------------------------------------------------------------

def _mx_bytes(rows, cols, fmt):
    return rows * _blocks(cols) * (FORMATS[fmt][4] + 1)


def work(case):
    kind = case["kind"]
    if kind in ("norm", "backward", "quantize", "dequantize"):
        n, es = case["rows"] * case["cols"], BYTES[case["dtype"]]
        if kind == "norm":
            out = n * es if case["out"] == "plain" else _mx_bytes(case["rows"], case["cols"], case["out"])
            return dict(bytes=n * es * (3 if case["residual"] else 1) + out + case["cols"] * es, flops=5 * n)
        if kind == "backward":
            return dict(bytes=n * es * (4 if case["stream"] else 3) + 2 * case["cols"] * es + 4 * case["rows"], flops=10 * n)
        if kind == "dequantize":
            return dict(bytes=_mx_bytes(case["rows"], case["cols"], case["format"]) + n * es, flops=n)
        written = (_mx_bytes(case["rows"], case["cols"], case["format"]) if case["axes"] != "columns" else 0) + (
            _mx_bytes(case["cols"], case["rows"], case["format"]) if case["axes"] != "rows" else 0)
        if case["format"] not in FLOAT8:  # and what they stand for
            written += n * es * (2 if case["axes"] == "both" else 1)
        return dict(bytes=n * es + written, flops=3 * n)
    m, n, k = case["m"], case["n"], case["k"]
    if kind == "train":
        es = BYTES[case["dtype"]]
        return dict(bytes=2 * es * (m * k + m * n + n * k), flops=6 * m * n * k)
    if kind == "layer":
        es = BYTES[case["dtype"]]
        return dict(bytes=3 * es * m * k + es * k + _mx_bytes(n, k, case["b"]) + es * m * n, flops=2 * m * n * k)
    es = BYTES[case["out"]]
    return dict(bytes=_mx_bytes(m, k, case["a"]) + _mx_bytes(n, k, case["b"]) + es * (m * n * (2 if case["residual"] else 1) + (n if case["bias"] else 0)),
                flops=2 * m * n * k)


def _exact_grid(fmt):
    """All values of a format that are not negative, ascending: an index is the code."""
    bits, low, high, top, _ = FORMATS[fmt]
    grid = [i * 2.0 ** (low - bits) for i in range(2 ** bits)]
    grid += [(1 + i / 2 ** bits) * 2.0 ** e for e in range(low, high + 1) for i in range(2 ** bits)]
    return torch.tensor([v for v in grid if v <= top], dtype=torch.float64, device="cuda")


def _exact_power(e):
    """2^e of whole numbers in float64."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_quantized(x, fmt):
    """(values, powers of two [row][block]) of x in float64: the nearest value of the grid, of two as near the one of even code."""
    grid = _exact_grid(fmt)
    rows, cols = x.shape
    filled = torch.zeros(rows, _blocks(cols) * 32, dtype=torch.float64, device=x.device)
    filled[:, :cols] = x
    filled = filled.view(rows, -1, 32)
    top = filled.abs().max(2).values
    floor = torch.floor(torch.log2(top.clamp(min=2.0 ** -200)))
    scale = _exact_power((floor - FORMATS[fmt][2]).clamp(min=-127))
    q = filled / scale[..., None]
    size = q.abs().clamp(max=float(grid[-1]))
    below = (torch.searchsorted(grid, size, right=True) - 1).clamp(max=grid.numel() - 2)
    down, up = size - grid[below], grid[below + 1] - size
    code = torch.where((up < down) | ((up == down) & (below % 2 == 1)), below + 1, below)
    return (grid[code] * torch.sign(q)).view(rows, -1), scale


def _exact_numbers(pair):
    values, scale = pair
    return values * scale.repeat_interleave(32, 1)


def _exact_operand(pair, fmt):
    """float64 values of a matrix as it lies in memory, from its codes."""
    codes, scales = pair
    if fmt in FLOAT8:
        sign, size = codes >= 128, codes & 127
    else:
        nibbles = torch.stack((codes % 16, codes // 16), 2).flatten(1)
        sign, size = nibbles >= 8, nibbles & 7
    values = _exact_grid(fmt)[size.long()]
    return _exact_numbers((torch.where(sign, -values, values), _exact_power(scales.t().long() - 127)))


def _e8m0(scale):
    return scale.t().contiguous()


def exact(case, seed):
    s, kind = _inputs(case, seed), case["kind"]
    if kind in ("norm", "layer"):
        h, stream = s["x"].double(), None
        if "residual" in s:
            stream = h + s["residual"].double()
            h = stream.to(s["x"].dtype).double()
        rstd = 1.0 / torch.sqrt((h * h).sum(1) / h.shape[1] + EPS)
        y = h * rstd[:, None] * (s["weight"].double() + case.get("offset", 0.0))
        if kind == "layer":
            return dict(stream=stream, c=_exact_numbers(_exact_quantized(y, case["format"])) @ _exact_operand(s["b"], case["b"]).t())
        if case["out"] == "plain":
            return dict(stream=stream, y=y, rstd=rstd)
        values, scale = _exact_quantized(y, case["out"])
        return dict(stream=stream, values=values, scales=_e8m0(scale))
    if kind == "backward":
        h, grad, r = s["h"].double(), s["grad"].double(), s["rstd"].double()[:, None]
        g = grad * (s["weight"].double() + case["offset"])
        # the derivative of h_i r(h) along h_j: r (1 at i = j) - h_i h_j r^3 / cols
        grad_x = r * g - h * (r ** 3 / h.shape[1]) * (g * h).sum(1, keepdim=True)
        if "stream" in s:
            grad_x = grad_x + s["stream"].double()
        return grad_x, (grad * h * r).sum(0)
    if kind == "quantize":
        found = {}
        for axis, m in (("rows", s["x"].double()), ("columns", s["x"].double().t().contiguous())):
            if case["axes"] in (axis, "both"):
                values, scale = _exact_quantized(m, case["format"])
                found[axis] = values if case["format"] in FLOAT8 else _exact_numbers((values, scale))[:, :m.shape[1]]
                found[axis + "_scales"] = _e8m0(scale)
        return found
    if kind == "dequantize":
        return _exact_operand(s["a"], case["format"])[:, :case["cols"]]
    if kind == "train":
        x, w, g = s["x"].double(), s["w"].double(), s["grad"].double()

        def product(a, a_format, b, b_format):
            return _exact_numbers(_exact_quantized(a, a_format)) @ _exact_numbers(_exact_quantized(b, b_format)).t()

        f, e = case["format"], case["gradients"]
        return dict(y=product(x, f, w, f), grad_x=product(g, e, w.t().contiguous(), f),
                    grad_w=product(g.t().contiguous(), e, x.t().contiguous(), f))
    c = _exact_operand(s["a"], case["a"]) @ _exact_operand(s["b"], case["b"]).t()
    if "bias" in s:
        c = c + s["bias"].double()
    if "residual" in s:
        c = c + s["residual"].double()
    return torch.relu(c) if case["relu"] else c
