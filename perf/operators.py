"""Eight-bit floating-point operators around the cut of a split network, one pass at a time: plain forms in torch, and the
framework's kernels.

A coded matrix is [rows, cols] 8-bit floating-point codes (E4M3 or E5M2) with a scale for each block of 128 columns of a row
(``row``) or for each 128 x 128 tile (``tile``); scales are binary32 (``f32``) or powers of two (``e8m0``).  An operator is one of
  quantize         a matrix -> codes and scales, as it stands or transposed           (``rans_block_quantize``)
  dequantize       codes and scales -> a matrix                                       (``rans_block_dequantize``)
  norm             residual added, root-mean-square norm, codes and scales            (``rans_norm_quantize``)
  norm_backward    the gradients of the last one's input and weight                   (``rans_norm_backward``)
  matmul           A B^T of two coded matrices                                        (``rans_block_matmul``)

Eight-bit values are returned as torch's eight-bit types, the scales beside them.
"""
import math

import torch

own = False

BLOCK = 128
DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
FORMATS = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
VMAX = {"e4m3": 448.0, "e5m2": 57344.0}
EPS = 1e-5


def listed():
    def quantize(name, rows, cols, dtype, fmt, scale, block, transpose=False, op="quantize"):
        return dict(name=name, op=op, rows=rows, cols=cols, dtype=dtype, fmt=fmt, scale=scale, block=block, transpose=transpose)

    def norm(name, op, rows, cols, dtype, scale):
        return dict(name=name, op=op, rows=rows, cols=cols, dtype=dtype, fmt="e4m3", scale=scale, residual=True)

    def matmul(name, m, n, k, out, fmt_a, fmt_b, scale, block_b):
        return dict(name=name, op="matmul", m=m, n=n, k=k, out=out, fmt_a=fmt_a, fmt_b=fmt_b, scale=scale, block_b=block_b, tight=False)

    return [
        # The hidden state of one token on its way to the other half of the network: latency.
        quantize("quantize_token", 1, 4096, "fp16", "e4m3", "e8m0", "row"),
        # A prefill batch's hidden states, 8 x 2048 tokens: bandwidth.
        quantize("quantize_hidden", 8 * 2048, 4096, "fp16", "e4m3", "e8m0", "row"),
        # The gradient of a ragged batch's output, along the tokens, for the weight's gradient.
        quantize("quantize_gradient_t", 11 * 1021, 4096, "bf16", "e5m2", "f32", "row", transpose=True),
        # Hidden states of 5120 channels arrive coded, in a request of 395 tokens and more.
        quantize("dequantize_hidden", 13 * 395, 5120, "bf16", "e4m3", "f32", "row", op="dequantize"),
        # Between two layers of a decoding step, eight sequences of one token.
        norm("norm_tokens", "norm", 8, 4096, "bf16", "f32"),
        # The same for a prefill batch.
        norm("norm_hidden", "norm", 8 * 2048, 4096, "fp16", "e8m0"),
        # Gradients of the norm for one request, and for a whole batch of training.
        norm("norm_backward_request", "norm_backward", 395, 5120, "bf16", "f32"),
        norm("norm_backward_hidden", "norm_backward", 8 * 2048, 4096, "bf16", "f32"),
        # The three projections of attention at once for a single token: the weights' bytes.
        matmul("matmul_token", 1, 3 * 4096, 4096, "bf16", "e4m3", "e4m3", "f32", "tile"),
        # The same for one request's ragged prompt.
        matmul("matmul_request", 395, 3 * 4096, 4096, "fp16", "e4m3", "e4m3", "f32", "tile"),
        # The same for a prefill batch: the matrix cores.
        matmul("matmul_prefill", 8 * 2048, 3 * 4096, 4096, "bf16", "e4m3", "e4m3", "e8m0", "tile"),
        # The weight's gradient of a square projection over a ragged batch of tokens.
        matmul("matmul_weight_gradient", 4096, 4096, 11 * 1021, "fp32", "e5m2", "e4m3", "f32", "row"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(("quantize", "dequantize", "norm", "norm_backward", "matmul", "matmul"))
    scale = rng.choice(("f32", "e8m0"))
    if op == "matmul":
        kind = rng.choice(("tokens", "prompt", "prompt", "gradient"))
        n, k = (rng.choice((96, 384, 1024, 4096, 5120, 12288, _log_int(rng, 65, 12288))) for _ in range(2))
        m = _log_int(rng, 1, 64) if kind == "tokens" else _log_int(rng, 65, 16384)
        if kind == "gradient":
            m, k = k, m
        while m * n * k > 16384 * 12288 * 4096:
            m = m // 2 + 1
        fmt_a, fmt_b = ("e5m2", "e4m3") if kind == "gradient" else ("e4m3", "e4m3")
        return dict(op=op, m=m, n=n, k=k, out="fp32" if kind == "gradient" else rng.choice(("bf16", "fp16", "fp32")), fmt_a=fmt_a,
                    fmt_b=fmt_b, scale=scale, block_b="row" if kind == "gradient" else rng.choice(("tile", "tile", "row")),
                    tight=rng.random() < 0.25)
    cols = rng.choice((96, 768, 1024, 4096, 5120, _log_int(rng, 65, 8192)))
    rows = _log_int(rng, 1, min(16384, (1 << 26) // cols))
    dtype = rng.choice(("bf16", "fp16", "fp32"))
    if dtype == "fp32":
        rows = rows // 2 + 1
    if op in ("norm", "norm_backward"):
        return dict(op=op, rows=rows, cols=cols, dtype=dtype, fmt=rng.choice(("e4m3", "e4m3", "e5m2")), scale=scale, residual=rng.random() < 0.75)
    return dict(op=op, rows=rows, cols=cols, dtype=dtype, fmt=rng.choice(("e4m3", "e4m3", "e5m2")), scale=scale,
                block=rng.choice(("row", "row", "tile")), transpose=op == "quantize" and rng.random() < 0.5)


def _up(n, to):
    return -(-n // to) * to


# ---------------------------------------------------------------- inputs


def _hidden(g, rows, cols):
    """Hidden states: unit normal, 1 % of the channels x20."""
    x = torch.randn(rows, cols, device="cuda", generator=g)
    x[:, torch.randperm(cols, device="cuda", generator=g)[: max(1, cols // 100)]] *= 20.0
    return x


def _buffers(rows, cols, scale, block):
    """Memory for a coded matrix: rows of codes 16 bytes apart or a multiple of it, rows of scales a multiple of four."""
    srows = -(-rows // BLOCK) if block == "tile" else rows
    return (torch.zeros(rows, _up(cols, 16), dtype=torch.uint8, device="cuda"),
            torch.zeros(srows, _up(-(-cols // BLOCK), 4), dtype=torch.uint8 if scale == "e8m0" else torch.float32, device="cuda"))


def _coded(x, fmt, scale, block, tight=False):
    """(codes, scales) of x as a program that received them holds them."""
    rows, cols = x.shape
    q, s = _quantize(x, fmt, scale, block)
    if tight:
        return q.view(torch.uint8).contiguous(), (s.view(torch.uint8) if scale == "e8m0" else s).contiguous()
    codes, scales = _buffers(rows, cols, scale, block)
    codes[:, :cols] = q.view(torch.uint8)
    scales[:, : s.shape[1]] = s.view(torch.uint8) if scale == "e8m0" else s
    return codes, scales


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    st = {"case": case}
    if case["op"] == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        st["a"], st["a_scale"] = _coded(_hidden(g, m, k), case["fmt_a"], case["scale"], "row", case["tight"])
        st["b"], st["b_scale"] = _coded(torch.randn(n, k, device="cuda", generator=g) * k ** -0.5, case["fmt_b"], case["scale"], case["block_b"], case["tight"])
        st["c"] = torch.empty(m, n, dtype=DTYPES[case["out"]], device="cuda")
        return st
    rows, cols, dtype = case["rows"], case["cols"], DTYPES[case["dtype"]]
    x = _hidden(g, rows, cols)
    if case["op"] == "quantize":
        st["x"] = x.to(dtype)
        st["codes"], st["scales"] = _buffers(*((cols, rows) if case["transpose"] else (rows, cols)), case["scale"], case["block"])
        return st
    if case["op"] == "dequantize":
        st["codes"], st["scales"] = _coded(x, case["fmt"], case["scale"], case["block"])
        st["x"] = torch.empty(rows, cols, dtype=dtype, device="cuda")
        return st
    st["weight"] = (1 + 0.1 * torch.randn(cols, device="cuda", generator=g)).to(dtype)
    other = torch.randn(rows, cols, device="cuda", generator=g).to(dtype) if case["residual"] else None
    if case["op"] == "norm":
        st["x"], st["residual"] = x.to(dtype), other
        st["sum"] = torch.empty(rows, cols, dtype=dtype, device="cuda")
        st["rstd"] = torch.empty(rows, dtype=torch.float32, device="cuda")
        st["codes"], st["scales"] = _buffers(rows, cols, case["scale"], "row")
        return st
    # what the forward pass left, the gradient of its output, and the one that comes down the residual stream
    st["sum"] = x.to(dtype)
    st["rstd"] = torch.rsqrt(st["sum"].float().square().mean(1) + EPS)
    st["dy"], st["dsum"] = torch.randn(rows, cols, device="cuda", generator=g).to(dtype), other
    st["dx"] = torch.empty(rows, cols, dtype=dtype, device="cuda")
    st["dweight"] = torch.empty(cols, dtype=torch.float32, device="cuda")
    return st


# ---------------------------------------------------------------- plain forms


def _blocks_of(x, block):
    """x padded with zeros, as [row blocks, rows of a block, column blocks, BLOCK]."""
    rows, cols = x.shape
    h = BLOCK if block == "tile" else 1
    x = torch.nn.functional.pad(x, (0, _up(cols, BLOCK) - cols, 0, _up(rows, h) - rows))
    return x.view(-1, h, x.shape[1] // BLOCK, BLOCK)


def _quantize(x, fmt, scale, block):
    rows, cols = x.shape
    v = _blocks_of(x.float(), block)
    a = v.abs()
    a = torch.where(a < math.inf, a, torch.zeros_like(a)).amax((1, 3))
    if scale == "e8m0":
        m, e = torch.frexp(a / VMAX[fmt] * 256)  # times 256: no subnormal number on the way
        e = torch.where(m > 0.5, e, e - 1) - 8
        s = torch.where(a > 0, e.clamp(min=-126) + 127, 127).to(torch.uint8).view(torch.float8_e8m0fnu).float()
    else:
        s = torch.where(a > 0, (a / VMAX[fmt]).clamp(min=2.0 ** -126), torch.ones_like(a))
    q = (v * (1 / s)[:, None, :, None]).to(FORMATS[fmt])
    q = q.view(torch.uint8).reshape(-1, v.shape[2] * BLOCK)[:rows, :cols].view(FORMATS[fmt])
    return q, s.to(torch.float8_e8m0fnu) if scale == "e8m0" else s


def _values(codes, scales, rows, cols, fmt, block):
    """The binary32 values of a coded matrix."""
    s = scales.view(torch.float8_e8m0fnu).float() if scales.dtype == torch.uint8 else scales
    s = s[:, : -(-cols // BLOCK)]
    if block == "tile":
        s = s.repeat_interleave(BLOCK, 0)[:rows]
    return codes[:, :cols].view(FORMATS[fmt]).float() * s.repeat_interleave(BLOCK, 1)[:, :cols]


def _plain(st):
    case = st["case"]
    if case["op"] == "matmul":
        a = _values(st["a"], st["a_scale"], case["m"], case["k"], case["fmt_a"], "row")
        b = _values(st["b"], st["b_scale"], case["n"], case["k"], case["fmt_b"], case["block_b"])
        return (a @ b.t()).to(DTYPES[case["out"]])
    if case["op"] == "quantize":
        return _quantize(st["x"].t() if case["transpose"] else st["x"], case["fmt"], case["scale"], case["block"])
    dtype = DTYPES[case["dtype"]]
    if case["op"] == "dequantize":
        return _values(st["codes"], st["scales"], case["rows"], case["cols"], case["fmt"], case["block"]).to(dtype)
    w = st["weight"].float()
    if case["op"] == "norm":
        h = st["x"] if st["residual"] is None else (st["x"].float() + st["residual"].float()).to(dtype)
        rstd = torch.rsqrt(h.float().square().mean(1) + EPS)
        return h, rstd, *_quantize(h.float() * rstd[:, None] * w, case["fmt"], case["scale"], "row")
    dy, xh = st["dy"].float(), st["sum"].float() * st["rstd"][:, None]
    gr = dy * w
    dx = st["rstd"][:, None] * (gr - xh * (gr * xh).mean(1, keepdim=True))
    if st["dsum"] is not None:
        dx = dx + st["dsum"].float()
    return dx.to(dtype), (dy * xh).sum(0)


# ---------------------------------------------------------------- the framework's kernels


def _layout(B, rows, cols, codes, scales, fmt, block):
    return B.make_blocks(rows, cols, codes.stride(0), scales.stride(0), B.E4M3 if fmt == "e4m3" else B.E5M2,
                         B.SCALE_E8M0 if scales.dtype == torch.uint8 else B.SCALE_F32, B.BLOCK_TILE if block == "tile" else B.BLOCK_ROW)


def _plan(st, B):
    """Layouts, parameters, workspace and views of the buffers, which a program keeps from its first call."""
    case = st["case"]
    if case["op"] == "matmul":
        a = _layout(B, case["m"], case["k"], st["a"], st["a_scale"], case["fmt_a"], "row")
        b = _layout(B, case["n"], case["k"], st["b"], st["b_scale"], case["fmt_b"], case["block_b"])
        rc, size = B.rans_matmul_workspace_bytes(a, b)
        assert rc == 0
        return a, b, {"fp32": B.F32, "fp16": B.F16, "bf16": B.BF16}[case["out"]], B.workspace(size)
    rows, cols = case["rows"], case["cols"]
    dtype = {"fp32": B.F32, "fp16": B.F16, "bf16": B.BF16}[case["dtype"]]
    if case["op"] in ("quantize", "dequantize"):
        shape = (cols, rows) if case["transpose"] else (rows, cols)
        return _layout(B, *shape, st["codes"], st["scales"], case["fmt"], case["block"]), dtype, _eight_bits(st, shape[1])
    p = B.make_norm_params(rows, cols, dtype, dtype, EPS)
    if case["op"] == "norm":
        return p, _layout(B, rows, cols, st["codes"], st["scales"], case["fmt"], "row"), _eight_bits(st, cols)
    rc, size = B.rans_norm_workspace_bytes(p)
    assert rc == 0
    return p, B.workspace(size)


def _own(st):
    from paper_2511_11664_amd import binding as B
    case, plan = st["case"], st.get("plan")
    if plan is None:
        plan = st["plan"] = _plan(st, B)
    if case["op"] == "matmul":
        a, b, out, ws = plan
        rc = B.rans_block_matmul(st["a"], st["a_scale"], a, st["b"], st["b_scale"], b, out, st["c"], case["n"], ws)
        assert rc == 0
        return st["c"]
    if case["op"] == "quantize":
        layout, dtype, eight_bits = plan
        rc = B.rans_block_quantize(st["x"], case["cols"], dtype, case["transpose"], st["codes"], st["scales"], layout)
        assert rc == 0
        return eight_bits
    if case["op"] == "dequantize":
        layout, dtype, _ = plan
        rc = B.rans_block_dequantize(st["codes"], st["scales"], layout, dtype, st["x"], case["cols"])
        assert rc == 0
        return st["x"]
    if case["op"] == "norm":
        p, layout, eight_bits = plan
        total = st["sum"] if case["residual"] else None
        rc = B.rans_norm_quantize(st["x"], st["residual"], st["weight"], p, total, st["rstd"], None, st["codes"], st["scales"], layout)
        assert rc == 0
        return st["sum"] if case["residual"] else st["x"], st["rstd"], *eight_bits
    p, ws = plan
    rc = B.rans_norm_backward(st["dy"], st["dsum"], st["sum"], st["weight"], st["rstd"], p, st["dx"], st["dweight"], ws)
    assert rc == 0
    return st["dx"], st["dweight"]


def _eight_bits(st, cols):
    """The state's codes and scales as torch's eight-bit types."""
    s = st["scales"][:, : -(-cols // BLOCK)]
    return st["codes"][:, :cols].view(FORMATS[st["case"]["fmt"]]), s.view(torch.float8_e8m0fnu) if s.dtype == torch.uint8 else s


def run(st):
    return _own(st) if own else _plain(st)


# ---------------------------------------------------------------- what a pass cannot do without


def _coded_bytes(rows, cols, scale, block):
    return rows * cols + (-(-rows // BLOCK) if block == "tile" else rows) * -(-cols // BLOCK) * (1 if scale == "e8m0" else 4)


def work(case):
    size = {"fp32": 4, "fp16": 2, "bf16": 2}
    if case["op"] == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": _coded_bytes(m, k, case["scale"], "row") + _coded_bytes(n, k, case["scale"], case["block_b"]) + size[case["out"]] * m * n,
                "flops": 2 * m * n * k}
    rows, cols = case["rows"], case["cols"]
    e = size[case["dtype"]] * rows * cols
    if case["op"] in ("quantize", "dequantize"):
        shape = (cols, rows) if case["transpose"] else (rows, cols)
        return {"bytes": e + _coded_bytes(*shape, case["scale"], case["block"]), "flops": (3 if case["op"] == "quantize" else 1) * rows * cols}
    w = size[case["dtype"]] * cols
    if case["op"] == "norm":  # without a residual the sum is the input itself and not written
        return {"bytes": (3 if case["residual"] else 1) * e + w + 4 * rows + _coded_bytes(rows, cols, case["scale"], "row"), "flops": 8 * rows * cols}
    return {"bytes": (4 if case["residual"] else 3) * e + w + 4 * rows + 4 * cols, "flops": 11 * rows * cols}


# ---------------------------------------------------------------- the definition in 64 bits


def _nearest8(v, fmt):
    """The nearest number of the format, ties to the even one: its exponent's step, no coarser than the format's, no finer than its subnormals'."""
    digits, least = (3, -6) if fmt == "e4m3" else (2, -14)
    _, e = torch.frexp(v)
    step = torch.exp2((torch.clamp(e - 1, min=least) - digits).double())
    return torch.round(v / step) * step


def _exact_codes(x, fmt, scale, block):
    """(codes' values, scales) of a 64-bit matrix, by its definition."""
    rows, cols = x.shape
    h = BLOCK if block == "tile" else 1
    nr, nc = -(-rows // h), -(-cols // BLOCK)
    full = x.new_zeros(nr * h, nc * BLOCK)
    full[:rows, :cols] = x
    top = full.abs().reshape(nr, h, nc, BLOCK).permute(0, 2, 1, 3).reshape(nr, nc, -1).max(2).values
    s = top / (448 if fmt == "e4m3" else 57344)
    if scale == "e8m0":
        p = torch.exp2(torch.round(torch.log2(s)))  # a power of two next to s
        s = torch.where(p < s, 2 * p, torch.where(p / 2 >= s, p / 2, p))
    s = torch.where(top > 0, s, torch.ones_like(s))
    each = s[:, None, :, None].expand(nr, h, nc, BLOCK).reshape(nr * h, nc * BLOCK)
    return _nearest8(full / each, fmt)[:rows, :cols], s


def _exact_values(codes, scales, rows, cols, fmt, block):
    v = codes[:, :cols].contiguous().view(FORMATS[fmt]).double()
    s = torch.exp2(scales.double() - 127) if scales.dtype == torch.uint8 else scales.double()
    i = torch.arange(rows, device="cuda") // (BLOCK if block == "tile" else 1)
    return v * s[i][:, torch.arange(cols, device="cuda") // BLOCK]


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "matmul":
        a = _exact_values(st["a"], st["a_scale"], case["m"], case["k"], case["fmt_a"], "row")
        return a @ _exact_values(st["b"], st["b_scale"], case["n"], case["k"], case["fmt_b"], case["block_b"]).t().contiguous()
    if case["op"] == "quantize":
        return _exact_codes(st["x"].double().t().contiguous() if case["transpose"] else st["x"].double(), case["fmt"], case["scale"], case["block"])
    if case["op"] == "dequantize":
        return _exact_values(st["codes"], st["scales"], case["rows"], case["cols"], case["fmt"], case["block"])
    w = st["weight"].double()
    if case["op"] == "norm":
        h = st["x"].double()
        if st["residual"] is not None:  # the sum is kept, and normed, in the stream's own type
            h = (h + st["residual"].double()).to(DTYPES[case["dtype"]]).double()
        rstd = 1 / ((h * h).mean(1) + EPS).sqrt()
        return h, rstd, *_exact_codes(h * rstd[:, None] * w, case["fmt"], case["scale"], "row")
    r, h, dy = st["rstd"].double()[:, None], st["sum"].double(), st["dy"].double()
    dx = r * (dy * w) - h * r ** 3 * (dy * w * h).sum(1, keepdim=True) / case["cols"]
    if st["dsum"] is not None:
        dx = dx + st["dsum"].double()
    return dx, (dy * h * r).sum(0)
