"""Microscaled 4-bit products and the root-mean-square norm with its 8-bit output, as they are measured.

A playback replays a sublayer of a language model at a lower precision: the norm over the residual stream, whose
output is rounded to 8 bits on the way (``norm``, backward ``norm_grad``), and linear layers whose operands are
rounded to 4-bit floating point with a scale for each short block (``quant``; their product ``matmul``; the whole
layer, from recorded tensors to results, ``linear``).

Definitions.  Operations are float32 ones, each rounded once, unless said otherwise.
  codes   a 4-bit value is one of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}; E2M1(x) is the nearest, ties to the even code,
          at most 6 in magnitude.  Two codes a byte, the first in the low half.
  mxfp4   blocks of 32 along the product's axis: e = floor(log2 max |x|) - 2, at least -127; values E2M1(x 2^-e) 2^e.
          The block's scale is the byte e + 127.
  nvfp4   blocks of 16, and a float32 scale for each row: t = 2688 / amax over the row, scale = amax / 2688; over the
          block b = E4M3(max |x t| / 6), the nearest 8-bit float of 3 mantissa bits; values E2M1((x t) (1 / b)) b scale.
          (Where b is 0 the block's are.)
  scales  the bytes of 128 rows by 4 blocks are together, 512 bytes: row r, block k at (r mod 32) 16 + (r div 32) 4 + k;
          such tiles in the order of the blocks, then of the rows.
  matmul  out[m, n] = (sum over k of a[m, k] b[n, k]) (sa[m] sb[n]) + bias[n].
  linear  forward: x by row times w by row. Backward, of g = dL/dout: dL/dx = g by row times w by column,
          dL/dw = g by column times x by column.
  norm    s = x + residual in the tensors' type; v = sum s^2 / n in 64 bits; rstd = 1 / sqrt(v + eps);
          y = (s rstd) weight.  8 bits: amax = max |y| over the row, scale = amax / 127, q the nearest integer of
          y (127 / amax); the values are q scale.
  norm_grad   with n = s rstd, g = dL/dy weight: dL/dx = rstd (g - n mean(g n)) + dL/ds, dL/dweight = sum over rows
          of dL/dy n.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
BLOCK = {"mxfp4": 32, "nvfp4": 16}
EPS = 1e-6


def listed():
    return [
        # the activation [8, 2048, 4096] by token, as the forward product takes it
        {"name": "quant_nv_tokens", "op": "quant", "format": "nvfp4", "axis": 0, "rows": 16384, "cols": 4096,
         "dtype": "bf16", "pad": 0},
        # a ragged batch by channel, as the weight gradient's product takes it
        {"name": "quant_mx_channels", "op": "quant", "format": "mxfp4", "axis": 1, "rows": 4099, "cols": 1024,
         "dtype": "f16", "pad": 0},
        # one token through a feed-forward weight
        {"name": "matmul_nv_token", "op": "matmul", "format": "nvfp4", "m": 1, "n": 4096, "k": 1024, "bias": True,
         "out": "bf16"},
        # a few sequences' tokens through a vocabulary of odd size: the weight's bytes bound it
        {"name": "matmul_mx_vocab_16", "op": "matmul", "format": "mxfp4", "m": 16, "n": 50257, "k": 1024, "bias": False,
         "out": "f16"},
        # a classifier's 1000 outputs of a ragged batch, a row of 129 blocks
        {"name": "matmul_nv_ragged", "op": "matmul", "format": "nvfp4", "m": 777, "n": 1000, "k": 2064, "bias": True,
         "out": "f32"},
        # the product of a training batch [8, 2048] in a feed-forward layer: the largest
        {"name": "matmul_mx_batch", "op": "matmul", "format": "mxfp4", "m": 16384, "n": 4096, "k": 1024, "bias": True,
         "out": "bf16"},
        # a layer's forward step from the recorded activation
        {"name": "linear_nv_forward", "op": "linear", "format": "nvfp4", "dir": "forward", "m": 2048, "n": 1024,
         "k": 4096, "dtype": "bf16"},
        # a layer's input and weight gradients from the recorded activation and output gradient
        {"name": "linear_mx_backward", "op": "linear", "format": "mxfp4", "dir": "backward", "m": 4096, "n": 4096,
         "k": 1024, "dtype": "bf16"},
        # one token's residual stream: all latency
        {"name": "norm_token", "op": "norm", "rows": 1, "cols": 1024, "dtype": "bf16", "weight": "bf16",
         "residual": True, "out": "values", "pad": 0},
        # a training batch's
        {"name": "norm_batch", "op": "norm", "rows": 16384, "cols": 4096, "dtype": "bf16", "weight": "f32",
         "residual": True, "out": "values", "pad": 0},
        # its gradients, with the residual stream's own gradient
        {"name": "norm_grad_batch", "op": "norm_grad", "rows": 16384, "cols": 4096, "dtype": "bf16", "weight": "f32",
         "stream": True, "pad": 0},
        # gradients of a few tokens of odd width
        {"name": "norm_grad_ragged", "op": "norm_grad", "rows": 77, "cols": 1001, "dtype": "f32", "weight": "f32",
         "stream": False, "pad": 0},
    ]


def _log(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    n = n | 1 if rng.random() < 0.4 and n < hi else n
    return min(max(n, lo), hi)


def draw(rng):
    """Another case: any operator, sizes over the whole range by their logarithm, odd ones and padded rows among
    them, every type and format; rows of any number of blocks for the products."""
    op = rng.choice(["quant", "quant", "matmul", "matmul", "matmul", "linear", "linear", "norm", "norm", "norm_grad"])
    dtype, format = rng.choice(["f32", "f16", "bf16"]), rng.choice(["mxfp4", "nvfp4"])
    if op == "quant":
        cols = _log(rng, 1, 16384)
        return {"op": op, "format": format, "axis": rng.choice([0, 1]), "rows": _log(rng, 1, min(50257, 60000000 // cols)),
                "cols": cols, "dtype": dtype, "pad": rng.choice([0, 0, 1, 8])}
    if op == "matmul":
        m, blocks = _log(rng, 1, 16384), _log(rng, 1, 16384 // BLOCK[format])
        k = blocks * BLOCK[format]
        most = min(60000000000 // (m * k), 60000000 // m, 300000000 // k, 50257)
        return {"op": op, "format": format, "m": m, "n": _log(rng, 1, max(1, most)), "k": k,
                "bias": rng.choice([False, True]), "out": dtype}
    if op == "linear":
        m, k = _log(rng, 1, 8192), _log(rng, 16, 8192)
        most = min(30000000000 // (m * k), 30000000 // m, 30000000 // k, 8192)
        return {"op": op, "format": format, "dir": rng.choice(["forward", "backward"]), "m": m,
                "n": _log(rng, 16, max(16, most)), "k": k, "dtype": dtype}
    cols = _log(rng, 1, 16384)
    case = {"op": op, "rows": _log(rng, 1, min(50257, 60000000 // cols)), "cols": cols, "dtype": dtype,
            "weight": rng.choice([dtype, "f32"]), "pad": rng.choice([0, 0, 1, 8])}
    if op == "norm":
        return {**case, "residual": rng.choice([True, True, False]), "out": rng.choice(["values", "values", "y"])}
    return {**case, "stream": rng.choice([True, False])}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _padded(x, pad):
    """x as the leading columns of a wider buffer."""
    if not pad:
        return x
    return torch.nn.functional.pad(x, (0, pad))[:, : x.shape[1]]


def _activation(rows, cols, dtype, gen, scale=1.0):
    """Normal values, tokens of different size, a few channels several times larger than the others."""
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    token = torch.exp(0.3 * torch.randn(rows, 1, generator=gen, device="cuda"))
    channel = torch.where(torch.rand(1, cols, generator=gen, device="cuda") < 0.01, 8.0, 1.0)
    return (x * token * channel * scale).to(DTYPES[dtype])


def _weight(n, dtype, gen):
    """A norm's weights, as training leaves them: around 1."""
    return (1.0 + 0.2 * torch.randn(n, generator=gen, device="cuda")).to(DTYPES[dtype])


def _inputs(case, seed):
    gen, op = _gen(seed), case["op"]
    if op == "quant":
        return {"x": _padded(_activation(case["rows"], case["cols"], case["dtype"], gen), case["pad"])}
    if op == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        a = _activation(m, k, "bf16", gen)
        w = (torch.randn(n, k, generator=gen, device="cuda") / math.sqrt(k)).to(torch.bfloat16)
        return {"a": _stored(a, case["format"]), "b": _stored(w, case["format"]),
                "bias": torch.randn(n, generator=gen, device="cuda") if case["bias"] else None}
    if op == "linear":
        m, n, k, dtype = case["m"], case["n"], case["k"], case["dtype"]
        return {"x": _activation(m, k, dtype, gen),
                "w": (torch.randn(n, k, generator=gen, device="cuda") / math.sqrt(k)).to(DTYPES[dtype]),
                "g": _activation(m, n, dtype, gen, scale=0.01)}
    rows, cols, dtype, pad = case["rows"], case["cols"], case["dtype"], case["pad"]
    got = {"x": _padded(_activation(rows, cols, dtype, gen), pad), "weight": _weight(cols, case["weight"], gen)}
    if op == "norm":
        # the layer's output, smaller than the stream that it is added to
        return {**got, "residual": _padded(_activation(rows, cols, dtype, gen, scale=3.0), pad) if case["residual"] else None}
    return {**got, "rstd": _rstd(got["x"]), "grad": _padded(_activation(rows, cols, dtype, gen, scale=0.01), pad),
            "stream": _padded(_activation(rows, cols, dtype, gen, scale=0.02), pad) if case["stream"] else None}


def _stored(x, format):
    """A matrix in 4 bits as a program holds it: packed codes, tiled block scales, the rows' scales (or None)."""
    code, block, scale = _codes(x.float(), format)
    rows, blocks = block.shape
    code = code.reshape(rows, -1)
    q = code[:, 0::2] | code[:, 1::2] << 4
    pad = -q.shape[1] % 16  # rows start on 16-byte boundaries
    q = torch.nn.functional.pad(q, (0, pad))[:, : q.shape[1]]
    tiles = torch.nn.functional.pad(block, (0, -blocks % 4, 0, -rows % 128))
    tiles = tiles.view(tiles.shape[0] // 128, 4, 32, tiles.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)
    return q, tiles, scale


def prepare(case, seed):
    """The tensors, a handle and the output buffers that the program reuses; a linear layer's weight is held in
    4 bits (both ways), as a program that replays the layer step after step holds it."""
    st = {"case": case, **_inputs(case, seed)}
    op = case["op"]
    if op == "linear":
        w = st["w"].float()
        st["wr"], st["wc"] = _rounded(w, case["format"]), _rounded(w.t(), case["format"])
    if own:
        import paper_2609_13544_gb300 as peat
        st["h"] = peat.Handle(0)
        if op == "quant":
            st["values"] = torch.empty(case["rows"], case["cols"], dtype=st["x"].dtype, device="cuda")
            st["scale"] = None
            if case["format"] == "nvfp4":
                st["scale"] = torch.empty(case["cols"] if case["axis"] else case["rows"], device="cuda")
        elif op == "matmul":
            st["a4"], st["b4"] = peat.Float4(case["format"], *st["a"]), peat.Float4(case["format"], *st["b"])
            st["out"] = torch.empty(case["m"], case["n"], dtype=DTYPES[case["out"]], device="cuda")
        elif op == "linear":
            st["layer"] = peat.Linear4(st["h"], st["w"], case["format"])
        else:
            like = lambda: torch.empty(case["rows"], case["cols"], dtype=st["x"].dtype, device="cuda")
            if op == "norm":
                st["sum"] = like() if case["residual"] else None
                st["out"], st["rstd"] = like(), torch.empty(case["rows"], device="cuda")
                st["scale"] = torch.empty(case["rows"], device="cuda") if case["out"] == "values" else None
            else:
                st["grad_x"], st["grad_weight"] = like(), torch.empty(case["cols"], device="cuda")
    return st


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _e2m1(x):
    """Codes of the nearest 4-bit values."""
    a = x.abs().clamp(max=6.0)
    n = torch.where(a < 2.0, torch.round(a * 2.0), torch.where(a < 4.0, torch.round(a) + 2.0, torch.round(a * 0.5) + 4.0))
    return torch.where(x < 0, n + 8.0, n).to(torch.uint8)


def _value(code):
    """The values of codes, from float 3 bits: exponent and one mantissa bit."""
    n = (code & 7).float()
    v = torch.where(n < 4.0, n * 0.5, torch.where(n < 6.0, n - 2.0, n * 2.0 - 8.0))
    return torch.where(code > 7, -v, v)


def _power(e):
    """2^e of int32 e from -127 to 127, by its bits."""
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).to(torch.int32).view(torch.float32)


def _e4m3(u):
    """The nearest 8-bit float of 3 mantissa bits and its byte, of 0 <= u <= 448."""
    step = _power(((u.view(torch.int32) >> 23) - 127).clamp(min=-6) - 3)
    v = (torch.round(u / step) * step).clamp(max=448.0)
    return v, ((v * 2.0 ** -120).view(torch.int32) >> 20).to(torch.uint8)


def _byte_value(byte):
    """The value of such a byte."""
    return (byte.to(torch.int32) << 20).view(torch.float32) * 2.0 ** 120


def _codes(x, format):
    """Codes [rows, blocks, block], the blocks' scale bytes and the rows' scales (mxfp4: None) of float32 rows."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, -cols % BLOCK[format])).view(rows, -1, BLOCK[format])
    if format == "mxfp4":
        e = ((x.abs().amax(2).view(torch.int32) >> 23) - 129).clamp(min=-127)
        return _e2m1(x * _power(-e)[:, :, None]), (e + 127).to(torch.uint8), None
    top = torch.full((rows,), 2688.0, device=x.device)  # (a division by a plain number multiplies by its reciprocal)
    amax = x.abs().amax((1, 2))
    t = top / amax
    use = torch.isfinite(t)
    y = x * torch.where(use, t, 0.0)[:, None, None]
    b, byte = _e4m3(y.abs().amax(2) / torch.full_like(y[:, :, 0], 6.0))
    r = torch.where(b > 0, 1.0 / b, 0.0)
    return _e2m1(y * r[:, :, None]), byte, torch.where(use, amax / top, 0.0)


def _factors(code, byte, scale, format):
    """(values without the rows' scales, those scales)."""
    rows = code.shape[0]
    f = _power(byte.to(torch.int32) - 127) if format == "mxfp4" else _byte_value(byte)
    return (_value(code) * f[:, :, None]).view(rows, -1), scale


def _rounded(x, format):
    return _factors(*_codes(x, format), format)


def _held(stored, format):
    """_factors of a matrix as it is stored."""
    q, tiles, scale = stored
    rows = q.shape[0]
    code = torch.stack([q & 15, q >> 4], 2).view(rows, -1, BLOCK[format])
    blocks = code.shape[1]
    t = tiles.view(-(-rows // 128), -(-blocks // 4), 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-(-rows // 128) * 128, -1)
    return _factors(code, t[:rows, :blocks], scale, format)


def _product(a, b, bias, dtype):
    (x, sa), (y, sb) = a, b
    out = x @ y.t()
    if sa is not None:
        out = out * (sa[:, None] * sb[None, :])
    return (out if bias is None else out + bias).to(dtype)


def _rstd(s):
    v = (s.double().square().sum(1) / s.shape[1]).float()
    return 1.0 / torch.sqrt(v + EPS)


def _plain(st):
    case, op = st["case"], st["case"]["op"]
    if op == "quant":
        x = st["x"].float()
        v, scale = _rounded(x.t() if case["axis"] else x, case["format"])
        v = v[:, : x.shape[0] if case["axis"] else x.shape[1]]
        v = v if scale is None else v * scale[:, None]
        return {"values": (v.t() if case["axis"] else v).to(st["x"].dtype).contiguous(),
                **({} if scale is None else {"scale": scale})}
    if op == "matmul":
        return _product(_held(st["a"], case["format"]), _held(st["b"], case["format"]), st["bias"], DTYPES[case["out"]])
    if op == "linear":
        dt, f = DTYPES[case["dtype"]], case["format"]
        if case["dir"] == "forward":
            return _product(_rounded(st["x"].float(), f), st["wr"], None, dt)
        return {"input": _product(_rounded(st["g"].float(), f), st["wc"], None, dt),
                "weight": _product(_rounded(st["g"].float().t(), f), _rounded(st["x"].float().t(), f), None, torch.float32)}
    x, w = st["x"], st["weight"].float()
    if op == "norm":
        s = x if st["residual"] is None else (x.float() + st["residual"].float()).to(x.dtype)
        rstd = _rstd(s)
        y = (s.float() * rstd[:, None]) * w
        got = {"rstd": rstd, **({} if st["residual"] is None else {"sum": s})}
        if case["out"] == "y":
            return {**got, "y": y.to(x.dtype)}
        amax = y.abs().amax(1)
        top = torch.full_like(amax, 127.0)
        r = top / amax
        use = torch.isfinite(r)
        scale = torch.where(use, amax / top, 0.0)
        q = torch.round(y * torch.where(use, r, 0.0)[:, None])
        return {**got, "values": (q * scale[:, None]).to(x.dtype), "scale": scale}
    n = x.float() * st["rstd"][:, None]
    d = st["grad"].float()
    g = d * w
    dx = st["rstd"][:, None] * (g - n * (g * n).mean(1, keepdim=True))
    dx = dx if st["stream"] is None else dx + st["stream"].float()
    return {"grad_x": dx.to(x.dtype), "grad_weight": (d * n).sum(0)}


def _own(st):
    import paper_2609_13544_gb300 as peat
    case, op, h = st["case"], st["case"]["op"], st["h"]
    if op == "quant":
        peat.peat_quantize_f4_raw(h, st["x"], case["format"], case["axis"], None, None, st["scale"], st["values"])
        return {"values": st["values"], **({} if st["scale"] is None else {"scale": st["scale"]})}
    if op == "matmul":
        peat.peat_matmul_f4_raw(h, st["a4"], st["b4"], st["out"], st["bias"])
        return st["out"]
    if op == "linear":
        if case["dir"] == "forward":
            return st["layer"].forward(st["x"])
        gx, gw = st["layer"].backward(st["g"], st["x"])
        return {"input": gx, "weight": gw}
    if op == "norm":
        got = {"rstd": st["rstd"], **({} if st["sum"] is None else {"sum": st["sum"]})}
        if case["out"] == "y":
            peat.peat_rmsnorm_raw(h, st["x"], st["weight"], EPS, residual=st["residual"], sum=st["sum"], y=st["out"],
                                  rstd=st["rstd"])
            return {**got, "y": st["out"]}
        peat.peat_rmsnorm_raw(h, st["x"], st["weight"], EPS, residual=st["residual"], sum=st["sum"], values=st["out"],
                              scale=st["scale"], rstd=st["rstd"])
        return {**got, "values": st["out"], "scale": st["scale"]}
    peat.peat_rmsnorm_backward_raw(h, st["grad"], st["x"], st["weight"], st["rstd"], st["grad_x"], st["grad_weight"],
                                   grad_sum=st["stream"])
    return {"grad_x": st["grad_x"], "grad_weight": st["grad_weight"]}


def run(st):
    """One pass through an operator."""
    return _own(st) if own else _plain(st)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def _bytes4(rows, k, format):
    """Of a matrix in 4 bits: codes, block scales, the rows' scales."""
    blocks = -(-k // BLOCK[format])
    return rows * blocks * (BLOCK[format] // 2 + 1) + (4 * rows if format == "nvfp4" else 0)


def work(case):
    op = case["op"]
    if op in ("matmul", "linear"):
        m, n, k, f = case["m"], case["n"], case["k"], case["format"]
        if op == "matmul":
            return {"bytes": _bytes4(m, k, f) + _bytes4(n, k, f) + (4 * n if case["bias"] else 0) + m * n * SIZE[case["out"]],
                    "flops": 2 * m * n * k}
        s = SIZE[case["dtype"]]
        if case["dir"] == "forward":
            return {"bytes": s * m * k + _bytes4(n, k, f) + s * m * n, "flops": 2 * m * n * k}
        return {"bytes": s * m * n + s * m * k + _bytes4(k, n, f) + s * m * k + 4 * n * k, "flops": 4 * m * n * k}
    n, s = case["rows"] * case["cols"], SIZE[case["dtype"]]
    if op == "quant":
        scales = 4 * (case["cols"] if case["axis"] else case["rows"]) if case["format"] == "nvfp4" else 0
        return {"bytes": 2 * n * s + scales, "flops": 4 * n}
    weight = case["cols"] * SIZE[case["weight"]]
    if op == "norm":
        return {"bytes": n * s * (4 if case["residual"] else 2) + weight + case["rows"] * (8 if case["out"] == "values" else 4),
                "flops": 6 * n}
    return {"bytes": n * s * (4 if case["stream"] else 3) + weight + 4 * case["rows"] + 4 * case["cols"], "flops": 9 * n}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _single(x):
    """Rounded to float32 (a float64 quotient, product or root of float32 values rounds to the float32 one)."""
    return x.to(torch.float32).to(torch.float64)


def _nearest4(x):
    """The nearest 4-bit values: by the borders between them, which belong to the neighbour of even code."""
    a, v = x.abs(), torch.zeros_like(x)
    for i in range(7):
        border = (LEVELS[i] + LEVELS[i + 1]) / 2
        v = torch.where(a >= border if i % 2 else a > border, LEVELS[i + 1], v)
    return torch.copysign(v, x)


def _two(e):
    """2^e in float64, by its bits (a power function may be off by a rounding)."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _rows4(x64, format):
    """Values (without the rows' scales) and the rows' scales of float64 rows that hold float32 values."""
    rows, cols = x64.shape
    wide = torch.zeros(rows, -(-cols // BLOCK[format]) * BLOCK[format], dtype=torch.float64, device=x64.device)
    wide[:, :cols] = x64
    wide = wide.unflatten(1, (-1, BLOCK[format]))
    if format == "mxfp4":
        peak = wide.abs().max(dim=2, keepdim=True).values
        s = _two((torch.frexp(peak).exponent - 3).clamp(min=-127))
        s = torch.where(peak > 0, s, 2.0 ** -127)
        return (_nearest4(wide / s) * s).flatten(1)[:, :cols], None
    peak = wide.abs().flatten(1).max(dim=1).values
    t = _single(2688.0 / peak)
    none = torch.isinf(t)
    y = _single(wide * torch.where(none, torch.zeros_like(t), t)[:, None, None])
    u = _single(y.abs().max(dim=2, keepdim=True).values / 6.0)
    b = u.to(torch.float32).to(torch.float8_e4m3fn).to(torch.float64)
    r = torch.where(b > 0, _single(1.0 / b), torch.zeros_like(b))
    return (_nearest4(_single(y * r)) * b).flatten(1)[:, :cols], torch.where(none, torch.zeros_like(peak), _single(peak / 2688.0))


def _matrix4(stored, format):
    """The float64 values of a stored matrix, its rows' scales among them."""
    q, tiles, scale = stored
    rows, blocks = q.shape[0], q.shape[1] * 2 // BLOCK[format]
    table = torch.tensor(LEVELS + [-v for v in LEVELS], dtype=torch.float64, device=q.device)
    code = torch.empty(rows, q.shape[1] * 2, dtype=torch.int64, device=q.device)
    code[:, 0::2], code[:, 1::2] = q % 16, q // 16
    r, k = torch.arange(rows, device=q.device)[:, None], torch.arange(blocks, device=q.device)[None, :]
    at = ((r // 128) * ((blocks + 3) // 4) + k // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + k % 4
    byte = tiles[at]
    f = _two(byte.to(torch.int64) - 127) if format == "mxfp4" else byte.view(torch.float8_e4m3fn).double()
    v = table[code] * f.repeat_interleave(BLOCK[format], dim=1)
    return v if scale is None else v * scale.double()[:, None]


def _times(a, b):
    (x, sx), (y, sy) = a, b
    out = torch.matmul(x, y.t())
    return out if sx is None else out * torch.outer(sx, sy)


def exact(case, seed):
    """What run returns for these inputs, in float64."""
    d, op = _inputs(case, seed), case["op"]
    if op == "quant":
        x = d["x"].double()
        v, s = _rows4(x.t().contiguous() if case["axis"] == 1 else x, case["format"])
        v = v if s is None else v * s[:, None]
        return {"values": v.t().contiguous() if case["axis"] == 1 else v, **({} if s is None else {"scale": s})}
    if op == "matmul":
        out = torch.matmul(_matrix4(d["a"], case["format"]), _matrix4(d["b"], case["format"]).t())
        return out if d["bias"] is None else out.add_(d["bias"].double())
    if op == "linear":
        x, w, g, f = d["x"].double(), d["w"].double(), d["g"].double(), case["format"]
        if case["dir"] == "forward":
            return _times(_rows4(x, f), _rows4(w, f))
        return {"input": _times(_rows4(g, f), _rows4(w.t(), f)), "weight": _times(_rows4(g.t(), f), _rows4(x.t(), f))}
    s, w = d["x"].double(), d["weight"].double()
    if op == "norm":
        if case["residual"]:
            s = (d["x"].double() + d["residual"].double()).to(torch.float32).to(d["x"].dtype).double()
        v = _single(torch.einsum("ij,ij->i", s, s) / case["cols"])
        # (a program passes eps as a float32)
        rstd = _single(1.0 / _single(torch.sqrt(_single(v + _single(torch.tensor(EPS, dtype=torch.float64))))))
        y = _single(_single(s * rstd[:, None]) * w)
        got = {"rstd": rstd, **({"sum": s} if case["residual"] else {})}
        if case["out"] == "y":
            return {**got, "y": y}
        peak = torch.maximum(y.max(dim=1).values, -y.min(dim=1).values)
        r = _single(127.0 / peak)
        none = torch.isinf(r)
        q = torch.round(_single(y * torch.where(none, torch.zeros_like(r), r)[:, None]))
        scale = torch.where(none, torch.zeros_like(peak), _single(peak / 127.0))
        return {**got, "values": q * scale[:, None], "scale": scale}
    rstd, dy = d["rstd"].double()[:, None], d["grad"].double()
    n, g = s * rstd, dy * w
    dx = rstd * (g - n * (torch.einsum("ij,ij->i", g, n) / case["cols"])[:, None])
    if case["stream"]:
        dx = dx + d["stream"].double()
    return {"grad_x": dx, "grad_weight": torch.einsum("ij,ij->j", dy, n)}
