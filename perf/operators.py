"""The 8-bit playback operators and the gradient list's norm, as they are measured.

A playback step in 8-bit integers replays a linear layer's recorded tensors (activation, weight, output
gradient) at a lower precision: every operand is rounded to 8-bit integers with one scale for each row or
each column (``quant``), the integer products give the forward output, the input gradient and the weight
gradient (``matmul``; ``linear`` is the whole layer, from recorded tensors to results), and the step ends, as
training does, with the norm over all gradient tensors and their clipping (``norm``, ``clip``).

Definitions.
  quant   amax = max |x| over the row (axis 0) or column (axis 1); scale = amax / 127 and r = 127 / amax, both
          float32 divisions; q = the nearest integer (ties to even) of the float32 product x r; the values are
          q scale. (A row whose r is not finite is zero; one that holds a NaN or an infinity has scale NaN.)
  matmul  out[m, n] = (sum over k of a[m, k] b[n, k]) sa[m] sb[n] + bias[n], the integer sum exact.
  linear  forward: x by row times w by row. Backward, of g = dL/dout: dL/dx = g by row times w by column,
          dL/dw = g by column times x by column.
  norm    per tensor and over all: the 2-norm of u g; the count of elements that are not finite.
  clip    the norm, c = min(1, limit / (norm + 1e-6)), and every tensor times u c.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def listed():
    return [
        # one token's activation: all latency
        {"name": "quant_f32_token", "op": "quant", "axis": 0, "rows": 1, "cols": 1024, "dtype": "f32", "pad": 0},
        # the activation [8, 2048, 4096] by channel, as the weight gradient's product takes it
        {"name": "quant_bf16_channels", "op": "quant", "axis": 1, "rows": 16384, "cols": 4096, "dtype": "bf16",
         "pad": 0},
        # one token through a feed-forward weight
        {"name": "matmul_token", "op": "matmul", "m": 1, "n": 4096, "k": 1024, "fill": "gauss", "bias": True,
         "out": "bf16", "pad": 0},
        # a few sequences' tokens through a vocabulary of odd size: the weight's bytes bound it
        {"name": "matmul_vocab_16", "op": "matmul", "m": 16, "n": 50257, "k": 1024, "fill": "gauss", "bias": False,
         "out": "f16", "pad": 0},
        # a classifier's 1000 outputs of a ragged batch, odd lengths throughout, full-range integers
        {"name": "matmul_ragged", "op": "matmul", "m": 777, "n": 1000, "k": 2049, "fill": "uniform", "bias": True,
         "out": "f32", "pad": 3},
        # a prompt's logits over the vocabulary
        {"name": "matmul_vocab_1024", "op": "matmul", "m": 1024, "n": 50257, "k": 1024, "fill": "gauss",
         "bias": False, "out": "f16", "pad": 0},
        # the product of a training batch [8, 2048] in a feed-forward layer: the largest
        {"name": "matmul_batch", "op": "matmul", "m": 16384, "n": 4096, "k": 1024, "fill": "gauss", "bias": True,
         "out": "bf16", "pad": 0},
        # a layer's forward step from the recorded activation
        {"name": "linear_forward", "op": "linear", "dir": "forward", "m": 2048, "n": 1024, "k": 4096,
         "dtype": "bf16"},
        # a layer's input and weight gradients from the recorded activation and output gradient
        {"name": "linear_backward", "op": "linear", "dir": "backward", "m": 4096, "n": 4096, "k": 1024,
         "dtype": "bf16"},
        # monitoring: the norms of a convolutional network's 161 gradient tensors
        {"name": "norm_f32_resnet50", "op": "norm", "list": "resnet50", "tensors": 161, "elements": 25557032,
         "dtype": "f32", "mixed": False, "packed": False, "unscale": 1.0,
         "size": 3.0},
        # clipping a language model's 292 gradient tensors
        {"name": "clip_bf16_gpt2", "op": "clip", "list": "gpt2_medium", "tensors": 292, "elements": 354823168,
         "dtype": "bf16", "mixed": False, "packed": False, "unscale": 1.0,
         "size": 3.0},
        # the biases and normalisation weights of a small layer, scaled half-precision gradients: the smallest list
        {"name": "clip_f16_vectors", "op": "clip", "list": "ragged", "tensors": 12, "elements": 9973, "dtype": "f16",
         "mixed": False, "packed": True, "unscale": 1.0 / 1024, "size": 3.0},
    ]


def _log(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    n = n | 1 if rng.random() < 0.4 and n < hi else n
    return min(max(n, lo), hi)


def draw(rng):
    """Another case: any operator, sizes over the whole range by their logarithm, odd ones and padded rows among
    them, every type, and, for the products, integers up to the largest sums."""
    op = rng.choice(["quant", "quant", "matmul", "matmul", "matmul", "linear", "linear", "norm", "clip", "clip"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if op == "quant":
        cols = _log(rng, 1, 16384)
        return {"op": op, "axis": rng.choice([0, 1]), "rows": _log(rng, 1, min(50257, 60000000 // cols)), "cols": cols,
                "dtype": dtype, "pad": rng.choice([0, 0, 1, 8])}
    if op == "matmul":
        m, k = _log(rng, 1, 16384), _log(rng, 1, 16384)
        most = min(60000000000 // (m * k), 60000000 // m, 300000000 // k, 50257)
        return {"op": op, "m": m, "n": _log(rng, 1, max(1, most)), "k": k,
                "fill": rng.choice(["gauss", "gauss", "uniform", "extreme"]), "bias": rng.choice([False, True]),
                "out": dtype, "pad": rng.choice([0, 0, 3, 16])}
    if op == "linear":
        m, k = _log(rng, 1, 8192), _log(rng, 16, 8192)
        most = min(30000000000 // (m * k), 30000000 // m, 30000000 // k, 8192)
        return {"op": op, "dir": rng.choice(["forward", "backward"]), "m": m, "n": _log(rng, 16, max(16, most)), "k": k,
                "dtype": dtype}
    return {"op": op, "list": "ragged", "tensors": rng.randint(1, 400), "elements": _log(rng, 1000, 300000000),
            "dtype": dtype, "mixed": rng.random() < 0.3, "packed": rng.random() < 0.5,
            "unscale": rng.choice([1.0, 1.0 / 1024]), "size": rng.choice([3.0, 3.0, 0.05])}


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


def _integers(rows, cols, fill, gen):
    if fill == "gauss":  # as quantised normal values come out
        return (torch.randn(rows, cols, generator=gen, device="cuda") * 32.0).round().clamp(-127, 127).to(torch.int8)
    if fill == "uniform":
        return torch.randint(-127, 128, (rows, cols), generator=gen, device="cuda", dtype=torch.int8)
    # almost all of one sign and size: the sums run up to their bound
    u = torch.rand(rows, cols, generator=gen, device="cuda")
    return torch.where(u < 0.97, 127, torch.where(u < 0.985, -127, 126)).to(torch.int8)


def _shapes(kind):
    if kind == "resnet50":
        got, cin = [(64, 3, 7, 7), (64,), (64,)], 64
        for width, blocks in ((64, 3), (128, 4), (256, 6), (512, 3)):
            for b in range(blocks):
                got += [(width, cin, 1, 1), (width,), (width,), (width, width, 3, 3), (width,), (width,),
                        (4 * width, width, 1, 1), (4 * width,), (4 * width,)]
                if b == 0:
                    got += [(4 * width, cin, 1, 1), (4 * width,), (4 * width,)]
                cin = 4 * width
        return got + [(1000, 2048), (1000,)]
    d, got = 1024, [(50257, 1024), (1024, 1024)]
    for _ in range(24):
        got += [(d,), (d,), (d, 3 * d), (3 * d,), (d, d), (d,), (d,), (d,), (d, 4 * d), (4 * d,), (4 * d, d), (d,)]
    return got + [(d,), (d,)]


def _sizes(case):
    if case["list"] != "ragged":
        return [math.prod(s) for s in _shapes(case["list"])]
    # many small tensors, a few large ones, some empty
    k = case["tensors"]
    w = [math.exp(2.5 * math.sin(12.9898 * (i + 1) + case["elements"])) if (i * 7 + case["elements"]) % 50 else 0.0
         for i in range(k)]
    total = sum(w) or 1.0
    got = [int(case["elements"] * v / total) for v in w]
    got[-1] += case["elements"] - sum(got)
    return got


def _places(case):
    """Each tensor's type and its place in the buffer of its type: behind one another ("packed"), or each on a
    boundary of 64 elements, as an allocator gives them."""
    got, at = [], {}
    for i, n in enumerate(_sizes(case)):
        dt = "f32" if case["mixed"] and i % 3 == 0 else case["dtype"]
        got.append((dt, at.get(dt, 0), n))
        at[dt] = at.get(dt, 0) + (n if case["packed"] else -(-n // 64) * 64)
    return got, at


def _buffers(case):
    """Zeroed buffers, one for each type, and the list's tensors in them."""
    places, at = _places(case)
    flat = {dt: torch.zeros(max(n, 1), dtype=DTYPES[dt], device="cuda") for dt, n in at.items()}
    return flat, [flat[dt][o : o + n] for dt, o, n in places]


def _gradients(case, seed):
    # "size": about a third of the norm over all, which clipping at 1 cuts or leaves
    gen = _gen(seed)
    flat, views = _buffers(case)
    loud = torch.exp(torch.randn(len(views), generator=gen, device="cuda")).tolist()
    for t, s in zip(views, loud):
        std = s * case["size"] / (case["unscale"] * math.sqrt(case["elements"]))
        t.copy_(torch.randn(t.numel(), generator=gen, device="cuda") * std)
    return views


def _inputs(case, seed):
    gen, op = _gen(seed), case["op"]
    if op == "quant":
        return {"x": _padded(_activation(case["rows"], case["cols"], case["dtype"], gen), case["pad"])}
    if op == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        return {"a": _padded(_integers(m, k, case["fill"], gen), case["pad"]),
                "b": _padded(_integers(n, k, case["fill"], gen), case["pad"]),
                "sa": torch.rand(m, generator=gen, device="cuda") * 0.02 + 0.005,
                "sb": torch.rand(n, generator=gen, device="cuda") * 0.001 + 0.0005,
                "bias": torch.randn(n, generator=gen, device="cuda") if case["bias"] else None}
    if op == "linear":
        m, n, k, dtype = case["m"], case["n"], case["k"], case["dtype"]
        return {"x": _activation(m, k, dtype, gen),
                "w": (torch.randn(n, k, generator=gen, device="cuda") / math.sqrt(k)).to(DTYPES[dtype]),
                "g": _activation(m, n, dtype, gen, scale=0.01)}
    return {"grads": _gradients(case, seed)}


def prepare(case, seed):
    """The tensors, a handle and the output buffers that the program reuses; a linear layer's weight is held in
    8 bits (both ways), as a program that replays the layer step after step holds it."""
    st = {"case": case, **_inputs(case, seed)}
    op = case["op"]
    if op == "linear":
        st["wr"], st["wc"] = _quant(st["w"], 0), _quant(st["w"], 1)
    elif op in ("norm", "clip"):
        st["flat"], st["outs"] = _buffers(case) if op == "clip" else (None, None)
    if own:
        import paper_2609_13544_gb300 as peat
        st["h"] = peat.Handle(0)
        if op == "quant":
            rows, cols = st["x"].shape
            st["values"] = torch.empty(rows, cols, dtype=st["x"].dtype, device="cuda")
            st["scale"] = torch.empty(cols if case["axis"] else rows, device="cuda")
        elif op == "matmul":
            st["out"] = torch.empty(case["m"], case["n"], dtype=DTYPES[case["out"]], device="cuda")
        elif op == "linear":
            st["layer"] = peat.Linear8(st["h"], st["w"])
        else:
            st["list"] = peat.GradList(st["grads"], st["outs"])
            st["record"] = torch.zeros(peat.GRADNORM_BYTES, dtype=torch.uint8, device="cuda")
            st["norms"] = torch.zeros(len(st["grads"]), device="cuda")
    return st


LIMIT = 1.0  # of the clipped norm


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _quant(x, axis):
    """(integers, scales): by row as they lie, by column transposed, so that the product's axis is the last."""
    x = x.float().t() if axis else x.float()
    amax = x.abs().amax(1)
    top = torch.full_like(amax, 127.0)  # (a division by a plain number multiplies by its reciprocal instead)
    r = top / amax
    use = torch.isfinite(r)
    q = torch.round(x * torch.where(use, r, 0.0)[:, None])
    return q.to(torch.int8).contiguous(), torch.where(use, amax / top, 0.0)


def _matmul(a, sa, b, sb, bias, dtype):
    out = (a.float() @ b.float().t()) * (sa[:, None] * sb[None, :])
    return (out if bias is None else out + bias).to(dtype)


def _norm(grads, unscale):
    sums = torch.stack([(t.float() * unscale).square().sum() for t in grads])
    bad = torch.stack([(~torch.isfinite(t)).sum() for t in grads]).sum()
    return sums.sum().sqrt(), sums.sqrt(), bad


def _plain(st):
    case, op = st["case"], st["case"]["op"]
    if op == "quant":
        q, scale = _quant(st["x"], case["axis"])
        v = q.float() * scale[:, None]
        return {"values": (v.t() if case["axis"] else v).to(st["x"].dtype).contiguous(), "scale": scale}
    if op == "matmul":
        return _matmul(st["a"], st["sa"], st["b"], st["sb"], st["bias"], DTYPES[case["out"]])
    if op == "linear":
        dt = DTYPES[case["dtype"]]
        if case["dir"] == "forward":
            return _matmul(*_quant(st["x"], 0), *st["wr"], None, dt)
        return {"input": _matmul(*_quant(st["g"], 0), *st["wc"], None, dt),
                "weight": _matmul(*_quant(st["g"], 1), *_quant(st["x"], 1), None, torch.float32)}
    norm, norms, bad = _norm(st["grads"], case["unscale"])
    if op == "norm":
        return {"norm": norm, "norms": norms, "bad": bad}
    c = torch.clamp(LIMIT / (norm + 1e-6), max=1.0)
    f = c * case["unscale"]
    _ = [out.copy_(t.float() * f) for t, out in zip(st["grads"], st["outs"])]
    return {"norm": norm, "coef": c, "norms": norms, "bad": bad, "clipped": st["flat"]}


def _record(record, norms):
    f = record.view(torch.float32)
    return {"norm": f[0], "coef": f[1], "norms": norms, "bad": record.view(torch.int64)[1]}


def _own(st):
    import paper_2609_13544_gb300 as peat
    case, op, h = st["case"], st["case"]["op"], st["h"]
    if op == "quant":
        peat.peat_quantize_i8_raw(h, st["x"], case["axis"], None, st["scale"], st["values"])
        return {"values": st["values"], "scale": st["scale"]}
    if op == "matmul":
        peat.peat_matmul_i8_raw(h, st["a"], st["sa"], st["b"], st["sb"], st["out"], st["bias"])
        return st["out"]
    if op == "linear":
        if case["dir"] == "forward":
            return st["layer"].forward(st["x"])
        gx, gw = st["layer"].backward(st["g"], st["x"])
        return {"input": gx, "weight": gw}
    if op == "norm":
        peat.peat_grad_norm_raw(h, st["list"], st["record"], st["norms"], unscale=case["unscale"])
        got = _record(st["record"], st["norms"])
        del got["coef"]
        return got
    peat.peat_grad_clip_raw(h, st["list"], LIMIT, st["record"], st["norms"], unscale=case["unscale"])
    return {**_record(st["record"], st["norms"]), "clipped": st["flat"]}


def run(st):
    """One pass through an operator."""
    return _own(st) if own else _plain(st)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "quant":
        n = case["rows"] * case["cols"]
        return {"bytes": 2 * n * SIZE[case["dtype"]] + 4 * (case["cols"] if case["axis"] else case["rows"]),
                "flops": 4 * n}
    if op == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": m * k + n * k + 4 * (m + n * (2 if case["bias"] else 1)) + m * n * SIZE[case["out"]],
                "flops": 2 * m * n * k}
    if op == "linear":
        m, n, k, s = case["m"], case["n"], case["k"], SIZE[case["dtype"]]
        if case["dir"] == "forward":
            return {"bytes": s * m * k + n * k + 4 * n + s * m * n, "flops": 2 * m * n * k}
        return {"bytes": s * m * n + s * m * k + n * k + 4 * k + s * m * k + 4 * n * k, "flops": 4 * m * n * k}
    sizes = _sizes(case)
    size = sum(n * (4 if case["mixed"] and i % 3 == 0 else SIZE[case["dtype"]]) for i, n in enumerate(sizes))
    if op == "norm":
        return {"bytes": size + 4 * len(sizes) + 16, "flops": 2 * sum(sizes)}
    return {"bytes": 2 * size + 4 * len(sizes) + 16, "flops": 3 * sum(sizes)}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _single(x):
    """Rounded to float32 (a float64 quotient or product of two float32 values rounds to the float32 one)."""
    return x.to(torch.float32).to(torch.float64)


def _whole(x64):
    """Integers (as float64) and scales of the rows of x64, whose values are float32."""
    peak = torch.maximum(x64.max(dim=1).values, -x64.min(dim=1).values)
    r = _single(127.0 / peak)
    none = torch.isinf(r)
    q = torch.round(_single(x64 * torch.where(none, torch.zeros_like(r), r).unsqueeze(1)))
    return q, torch.where(none, torch.zeros_like(peak), _single(peak / 127.0))


def _products(qa, sa, qb, sb):
    return torch.matmul(qa, qb.t()) * torch.outer(sa, sb)


def exact(case, seed):
    """What run returns for these inputs, in float64."""
    d, op = _inputs(case, seed), case["op"]
    if op == "quant":
        x = d["x"].double()
        q, s = _whole(x.t().contiguous() if case["axis"] == 1 else x)
        v = q * s.unsqueeze(1)
        return {"values": v.t().contiguous() if case["axis"] == 1 else v, "scale": s}
    if op == "matmul":
        out = _products(d["a"].double(), d["sa"].double(), d["b"].double(), d["sb"].double())
        return out if d["bias"] is None else out.add_(d["bias"].double())
    if op == "linear":
        x, w, g = d["x"].double(), d["w"].double(), d["g"].double()
        if case["dir"] == "forward":
            return _products(*_whole(x), *_whole(w))
        return {"input": _products(*_whole(g), *_whole(w.t().contiguous())),
                "weight": _products(*_whole(g.t().contiguous()), *_whole(x.t().contiguous()))}
    norms = torch.stack([torch.linalg.vector_norm(t.double()) * case["unscale"] for t in d["grads"]])
    norm = torch.linalg.vector_norm(norms)
    got = {"norm": norm, "norms": norms, "bad": torch.zeros((), dtype=torch.int64)}
    if op == "norm":
        return got
    c = torch.clamp(LIMIT / (norm + 1e-6), max=1.0)
    places, at = _places(case)
    flat = {dt: torch.zeros(max(n, 1), dtype=torch.float64, device="cuda") for dt, n in at.items()}
    for (dt, o, n), t in zip(places, d["grads"]):
        flat[dt][o : o + n] = t.double() * (c * case["unscale"])
    return {**got, "coef": c, "clipped": flat}
