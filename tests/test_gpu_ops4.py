"""The 4-bit products and the root-mean-square norm against their definitions in 64 bits.

Tolerances.  Codes, block scales, scales and values are defined by single float32 roundings that binary64 reproduces, so
they have to be equal; so do a norm's outputs, once the mean of squares (a 64-bit sum, rounded once) is.  The kernel sums
it with the rounding errors kept, to 2^-40: rows whose mean lies within that of a border between two float32 numbers are
left out (none or next to none).

A product's sum is added up in float32 block by block: a block's own sum is exact, at most K / block + K / 64 additions
are off by 2^-23 of what the sum can have reached, the sum S of the products' magnitudes; scaling and bias are four more
roundings.  16-bit outputs are off by half a step besides (2^-9 relative for bfloat16, 2^-12 for binary16, or half of the
smallest step).

A norm's gradients: n, g and the result take five roundings of 2^-24; c sums a row, at most 32 + cols / 256 products one
after the other and 20 partial sums, the weight's gradient at most rows / 400 + 64 rows, each addition off by 2^-24 of the
sum of magnitudes.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
BLOCK = {"mxfp4": 32, "nvfp4": 16}
LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
FORMATS = ["mxfp4", "nvfp4"]
DTYPES = ["f32", "f16", "bf16"]


@pytest.fixture(scope="module")
def h(peat_gpu):
    handle = peat_gpu.Handle(0)
    yield handle
    handle.close()


def dt(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def rng(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def same_bits(a, b):
    import torch
    v = {1: torch.int8, 2: torch.int16, 4: torch.int32}[a.element_size()]
    a, b = a.contiguous(), b.contiguous()
    both = torch.isnan(a) & torch.isnan(b) if a.is_floating_point() else torch.zeros_like(a, dtype=torch.bool)
    return bool(((a.view(v) == b.view(v)) | both).all())


def same_values(a, b):
    """Equal numbers (zeros of either sign), NaN where NaN."""
    import torch
    return a.shape == b.shape and bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all())


def single(x):
    return x.float().double()


def two(e):
    import torch
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


# ---------------------------------------------------------------------------
# rounding
# ---------------------------------------------------------------------------
def nearest(x):
    """Codes (without signs) of the nearest 4-bit values: a border belongs to the even code."""
    import torch
    a, n = x.abs(), torch.zeros(x.shape, dtype=torch.int64, device=x.device)
    for i in range(7):
        border = (LEVELS[i] + LEVELS[i + 1]) / 2
        n = torch.where(a >= border if i % 2 else a > border, i + 1, n)
    return n


def definition(x, format, axis):
    """(codes without signs [R, K], block scales' bytes [R, blocks], scale or None, float32 values [rows, cols])."""
    import torch
    v = x.double().t() if axis else x.double()
    R, K = v.shape
    B = BLOCK[format]
    wide = torch.zeros(R, -(-K // B) * B, dtype=torch.float64, device=x.device)
    wide[:, :K] = v
    w = wide.view(R, -1, B)
    if format == "mxfp4":
        bad = ~torch.isfinite(w).all(2)
        w = torch.where(bad[:, :, None], 0.0, w)
        amax = w.abs().amax(2)
        e = torch.where(amax > 0, torch.frexp(amax).exponent - 3, -127).clamp(min=-127)
        n = nearest(w * two(-e)[:, :, None])
        byte = torch.where(bad, 255, e + 127)
        f = torch.where(bad, float("nan"), two(e))
        val = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)[n] * f[:, :, None]
        scale = None
    else:
        bad = ~torch.isfinite(v).all(1)
        w = torch.where(bad[:, None, None], 0.0, w)
        amax = w.abs().amax((1, 2))
        t = (2688.0 / amax).float()
        none = ~torch.isfinite(t) | bad
        t = torch.where(none, 0.0, t)
        scale = torch.where(bad, float("nan"), torch.where(none, 0.0, (amax / 2688.0).float()))
        y = single(w * t.double()[:, None, None])
        b = single(y.abs().amax(2) / 6.0).float().to(torch.float8_e4m3fn)
        r = torch.where(b.float() > 0, 1.0 / b.double(), 0.0)
        n = nearest(single(y * single(r)[:, :, None]))
        byte = b.view(torch.uint8).int()
        val = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)[n] * b.double()[:, :, None]
        val = val * scale.double()[:, None, None]
    val = (torch.where(w < 0, -val, val)).view(R, -1)[:, :K].float()
    return n.view(R, -1), byte, scale, (val.t() if axis else val)


def untiled(P, block_scale, rows, blocks):
    s = block_scale.view(-(-rows // 128), -(-blocks // 4), 32, 4, 4).permute(0, 3, 2, 1, 4)
    s = s.reshape(-(-rows // 128) * 128, -1)
    return s[:rows, :blocks], s


def check_quant(P, h, x, format, axis, qpad=0, vpad=0, stream=None):
    import torch
    rows, cols = x.shape
    R, K = (cols, rows) if axis else (rows, cols)
    blocks = -(-K // BLOCK[format])
    width = blocks * BLOCK[format] // 2
    ld = (width + 15) // 16 * 16 + qpad
    qbuf = torch.full((R + 1, ld), 99, dtype=torch.uint8, device="cuda")
    vbuf = torch.full((rows + 1, cols + vpad), 7.0, dtype=x.dtype, device="cuda")
    q, v = qbuf[:R, :width], vbuf[:rows, :cols]
    bs = torch.full((P.f4_scale_bytes(R, blocks) + 5,), 77, dtype=torch.uint8, device="cuda")
    scale = torch.full((R,), -1.0, device="cuda") if format == "nvfp4" else None
    P.peat_quantize_f4_raw(h, x, format, axis, q, bs, scale, v, stream)
    torch.cuda.synchronize()
    en, eb, es, ev = definition(x, format, axis)
    code = torch.stack([q & 15, q >> 4], 2).view(R, -1)
    assert torch.equal((code & 7).long(), en)
    signs = torch.zeros_like(en, dtype=torch.bool)
    signs[:, :K] = (x.t() if axis else x) < 0
    assert bool(((code > 7) == signs)[en > 0].all())
    here, padded = untiled(P, bs[:-5], R, blocks)
    assert torch.equal(here.int(), eb.int())
    margin = padded.clone()
    margin[:R, :blocks] = 0
    assert not bool(margin.any()) and bool((bs[-5:] == 77).all())
    if scale is not None:
        assert same_bits(scale, es)
    assert same_values(v, ev.to(x.dtype))
    assert bool((qbuf[R:] == 99).all()) and bool((qbuf[:, width:] == 99).all())
    assert bool((vbuf[rows:] == 7).all()) and bool((vbuf[:, cols:] == 7).all())
    # each output alone gives the same
    v2 = torch.empty(rows, cols, dtype=x.dtype, device="cuda")
    P.peat_quantize_f4_raw(h, x, format, axis, None, None, None, v2, stream)
    torch.cuda.synchronize()
    assert same_values(v2, v)
    f = P.Float4(format, q, bs[:-5], scale)
    assert same_values(f.values()[:, :K].to(x.dtype), (v.t() if axis else v))


SHAPES = [(1, 1), (1, 1024), (3, 17), (5, 1000), (64, 64), (130, 257), (9, 2056), (7, 4096), (2, 16384), (3, 20000),
          (1000, 129), (4099, 40), (513, 72)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("format", FORMATS)
@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("shape", SHAPES)
def test_quantize(peat_gpu, h, dtype, format, axis, shape):
    import torch
    rows, cols = shape
    g = rng(rows * 31 + cols)
    for pad, off, qpad, vpad in ((0, 0, 0, 0), (8, 0, 16, 8), (3, 1, 32, 1)):
        buf = torch.randn(rows * (cols + pad) + off, generator=g, device="cuda")
        buf = (buf * torch.exp(2 * torch.randn(buf.shape, generator=g, device="cuda"))).to(dt(dtype))
        x = buf[off:].view(rows, cols + pad)[:, :cols]
        check_quant(peat_gpu, h, x, format, axis, qpad, vpad)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("format", FORMATS)
@pytest.mark.parametrize("axis", [0, 1])
def test_quantize_extremes(peat_gpu, h, dtype, format, axis):
    """Rows of zeros and negative zeros, the type's largest and smallest values, ties, NaN and infinities."""
    import torch
    big, tiny = torch.finfo(dt(dtype)).max, torch.finfo(dt(dtype)).smallest_normal
    sub = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}[dtype]
    x = torch.randn(14, 300, generator=rng(1), device="cuda")
    x[0] = 0.0
    x[1] = -0.0
    x[2] = torch.where(x[2] > 0, big, -big)
    x[3] = torch.where(x[3] > 0, tiny, -tiny)
    x[4] = torch.where(x[4] > 0, sub, -sub)
    x[5] = torch.randint(-24, 25, (300,), generator=rng(2), device="cuda") / 4.0  # borders between codes
    x[6, 70] = float("nan")
    x[7, 299] = float("inf")
    x[8, 0] = float("-inf")
    x[9] *= torch.where(torch.arange(300, device="cuda") % 2 == 0, 1.0, 2.0 ** -20)
    x[10] = 0.0
    x[10, 33] = big
    x[11] = 4e-38 if dtype != "f16" else 6e-5
    x[12] = torch.exp2(torch.arange(300, device="cuda") / 10.0 - 15)
    x = x.to(dt(dtype))
    check_quant(peat_gpu, h, x if axis == 0 else x.t().contiguous(), format, axis)
    check_quant(peat_gpu, h, x if axis == 1 else x.t().contiguous(), format, axis)


@pytest.mark.parametrize("format", FORMATS)
def test_quantize_of_nothing(peat_gpu, h, format):
    import torch
    for rows, cols in ((0, 5), (5, 0), (0, 0)):
        x = torch.empty(rows, cols, device="cuda")
        for axis in (0, 1):
            f = peat_gpu.peat_quantize_f4(h, x, format, axis)
            assert f.rows == (cols if axis else rows) and f.cols == 0 or f.rows == 0
            if f.scale is not None:
                assert bool((f.scale == 0).all())


def test_quantize_refusals(peat_gpu, h):
    import torch
    P, x = peat_gpu, torch.zeros(4, 40, device="cuda")
    q, bs = torch.zeros(4, 32, dtype=torch.uint8, device="cuda"), torch.zeros(1024, dtype=torch.uint8, device="cuda")
    sc = torch.zeros(4, device="cuda")
    for call in (lambda: P.peat_quantize_f4_raw(h, x, "fp4", 0, q, bs), lambda: P.peat_quantize_f4(h, x[0]),
                 lambda: P.peat_quantize_f4_raw(h, x, "mxfp4", 0, q[:, :16], bs),
                 lambda: P.peat_quantize_f4_raw(h, x, "mxfp4", 0, q.to(torch.int8), bs),
                 lambda: P.peat_quantize_f4_raw(h, x, "mxfp4", 0, q, bs[:100]),
                 lambda: P.peat_quantize_f4_raw(h, x.cpu(), "mxfp4", 0, q, bs),
                 lambda: P.peat_quantize_f4_raw(h, x, "nvfp4", 0, None, None, sc[:3], x),
                 lambda: P.peat_quantize_f4_raw(h, x.t(), "mxfp4", 0, None, None, None, x.t())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        P.peat_quantize_f4(h, x.double())
    for call in (lambda: P.peat_quantize_f4_raw(h, x, "mxfp4", 0), lambda: P.peat_quantize_f4_raw(h, x, "mxfp4", 2, None, None, None, x),
                 lambda: P.peat_quantize_f4_raw(h, x, "mxfp4", 0, q), lambda: P.peat_quantize_f4_raw(h, x, "mxfp4", 0, q, bs, sc),
                 lambda: P.peat_quantize_f4_raw(h, x[:, :32], "mxfp4", 0, torch.zeros(4, 24, dtype=torch.uint8, device="cuda")[:, :16], bs)):
        with pytest.raises(P.PeatError) as e:
            call()
        assert e.value.status == 1


# ---------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------
def random_f4(P, rows, K, format, g, spread=1.0):
    """A matrix in 4 bits of random codes and scales around 1, rows' scales too."""
    import torch
    blocks = K // BLOCK[format]
    ld = (K // 2 + 15) // 16 * 16
    q = torch.randint(0, 256, (rows, ld), generator=g, device="cuda", dtype=torch.uint8)[:, : K // 2]
    mid, off = (127, 6) if format == "mxfp4" else (56, 24)
    s = (mid + spread * torch.randint(-off, off + 1, (-(-rows // 128) * 128, -(-blocks // 4) * 4), generator=g,
                                      device="cuda")).to(torch.uint8)
    s[rows:] = 0
    s[:, blocks:] = 0
    tiles = s.view(-(-rows // 128), 4, 32, -(-blocks // 4), 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)
    scale = torch.rand(rows, generator=g, device="cuda") + 0.5 if format == "nvfp4" else None
    return P.Float4(format, q, tiles, scale)


def values64(f):
    """The float64 values of a Float4, by a route of its own."""
    import torch
    table = torch.tensor(LEVELS + [-v for v in LEVELS], dtype=torch.float64, device="cuda")
    code = torch.empty(f.rows, f.cols, dtype=torch.int64, device="cuda")
    code[:, 0::2], code[:, 1::2] = (f.q % 16).long(), (f.q // 16).long()
    B = BLOCK[f.format]
    blocks = f.cols // B
    r, k = torch.arange(f.rows, device="cuda")[:, None], torch.arange(blocks, device="cuda")[None, :]
    byte = f.block_scale[((r // 128) * ((blocks + 3) // 4) + k // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + k % 4]
    s = two(byte.long() - 127) if f.format == "mxfp4" else byte.view(torch.float8_e4m3fn).double()
    v = table[code] * s.repeat_interleave(B, 1)
    return v if f.scale is None else v * f.scale.double()[:, None]


def check_product(got, a, b, K, format, bias=None):
    """got against the float64 operands' product."""
    import torch
    exact, size = a @ b.t(), a.abs() @ b.abs().t()
    steps = K // BLOCK[format] + K // 64 + 2
    tol = size * steps * 2.0 ** -23 + 4 * EPS * size
    if bias is not None:
        exact, tol = exact + bias.double(), tol + EPS * (exact.abs() + bias.double().abs()) * 2
    if got.dtype != torch.float32:
        fi = torch.finfo(got.dtype)
        tol = tol + (exact.abs() + tol) * fi.eps / 2 + fi.smallest_normal * fi.eps / 2
    err = (got.double() - exact).abs()
    assert bool((err <= tol).all()), (float((err - tol).max()), float((err / tol.clamp(min=1e-300)).max()))


PRODUCTS = [(1, 1, 32), (1, 4096, 1024), (2, 130, 64), (16, 1000, 96), (17, 300, 2048), (33, 129, 4128), (100, 257, 160),
            (128, 128, 256), (129, 128, 512), (177, 50, 320), (192, 640, 1056), (193, 64, 288), (200, 1000, 2080), (256, 256, 8192),
            (300, 65, 1024), (777, 1000, 2080), (1025, 513, 32), (2000, 190, 736), (130, 20000, 512), (20000, 17, 480)]


@pytest.mark.parametrize("format", FORMATS)
@pytest.mark.parametrize("mnk", PRODUCTS)
def test_matmul(peat_gpu, h, format, mnk):
    import torch
    M, N, K = mnk
    K = K if format == "mxfp4" else K - 16 * (K // 32 % 2)  # (rows of whole 16-byte units, and of half ones)
    g = rng(M + 3 * N + 7 * K)
    a, b = random_f4(peat_gpu, M, K, format, g), random_f4(peat_gpu, N, K, format, g)
    x, y = values64(a), values64(b)
    bias = torch.randn(N, generator=g, device="cuda") * K ** 0.5
    for bv, out in ((None, "f32"), (bias, "bf16"), (bias, "f16")):
        got = peat_gpu.peat_matmul_f4(h, a, b, bv, dt(out))
        if out == "f16":  # (within its range)
            fits = (x @ y.t()).abs().max() < 3e4
            if not bool(fits):
                continue
        check_product(got, x, y, K, format, bv)
    # rows of the output at distances of their own, off the 16-byte grid
    for ldo, off in ((N + 3, 1), (N + 8, 0)):
        buf = torch.full((M * ldo + off,), 7.0, device="cuda", dtype=torch.bfloat16)
        view = buf[off:].view(M, ldo)
        peat_gpu.peat_matmul_f4_raw(h, a, b, view[:, :N], None)
        check_product(view[:, :N], x, y, K, format)
        assert bool((view[:, N:] == 7).all()) and bool((buf[:off] == 7).all())


@pytest.mark.parametrize("format", FORMATS)
def test_matmul_is_exact_where_float32_is(peat_gpu, h, format):
    """Sums that float32 holds whatever the order: equal to the 64-bit ones."""
    import torch
    g = rng(5)
    for M, N, K in ((64, 100, 1024), (300, 200, 4096)):
        a, b = random_f4(peat_gpu, M, K, format, g), random_f4(peat_gpu, N, K, format, g)
        one = 127 if format == "mxfp4" else 56
        for f in (a, b):
            f.block_scale.copy_(torch.where(f.block_scale > 0, one, 0))
            if f.scale is not None:
                f.scale.fill_(1.0)
        assert torch.equal(peat_gpu.peat_matmul_f4(h, a, b).double(), values64(a) @ values64(b).t())


@pytest.mark.parametrize("format", FORMATS)
def test_matmul_same_bits_each_call(peat_gpu, h, format):
    import torch
    g = rng(6)
    for M, N, K in ((7, 3000, 2048), (600, 700, 2048)):
        a, b = random_f4(peat_gpu, M, K, format, g), random_f4(peat_gpu, N, K, format, g)
        first = peat_gpu.peat_matmul_f4(h, a, b)
        for _ in range(5):
            assert same_bits(peat_gpu.peat_matmul_f4(h, a, b), first)


@pytest.mark.parametrize("format", FORMATS)
def test_matmul_of_nothing(peat_gpu, h, format):
    """No k: zeros, plus the bias."""
    import torch
    for M, N in ((3, 300), (300, 77)):
        a = peat_gpu.peat_quantize_f4(h, torch.empty(M, 0, device="cuda"), format)
        b = peat_gpu.peat_quantize_f4(h, torch.empty(N, 0, device="cuda"), format)
        bias = torch.randn(N, generator=rng(M), device="cuda")
        assert torch.equal(peat_gpu.peat_matmul_f4(h, a, b, bias), bias.expand(M, N))
        assert not bool(peat_gpu.peat_matmul_f4(h, a, b).any())
    empty = peat_gpu.peat_quantize_f4(h, torch.empty(0, 64, device="cuda"), format)
    some = peat_gpu.peat_quantize_f4(h, torch.ones(5, 64, device="cuda"), format)
    assert peat_gpu.peat_matmul_f4(h, empty, some).shape == (0, 5) and peat_gpu.peat_matmul_f4(h, some, empty).shape == (5, 0)


@pytest.mark.parametrize("format", FORMATS)
@pytest.mark.parametrize("axes", [(0, 0), (0, 1), (1, 0), (1, 1)])
@pytest.mark.parametrize("mnk", [(1, 40, 33), (5, 300, 1000), (64, 64, 64), (300, 513, 257), (600, 260, 2111)])
def test_product(peat_gpu, h, format, axes, mnk):
    """Operands rounded on the way, off the 16-byte grid and on it, of every type: those of the two calls."""
    import torch
    M, N, K = mnk
    g = rng(M + N + K)
    for pad, t in ((0, "bf16"), (3, "f32"), (8, "f16")):
        ops, held = [], []
        for rows, axis in ((M, axes[0]), (N, axes[1])):
            shape = (K, rows) if axis else (rows, K)
            x = torch.randn(shape[0], shape[1] + pad, generator=g, device="cuda").to(dt(t))[:, : shape[1]]
            ops.append(x)
            held.append(peat_gpu.peat_quantize_f4(h, x, format, axis))
        want = peat_gpu.peat_matmul_f4(h, *held, None, dt(t))
        check_product(want, values64(held[0]), values64(held[1]), held[0].cols, format)
        assert same_bits(peat_gpu.peat_product_f4(h, *ops, format, *axes, None, dt(t)), want)
        # one of them held already
        assert same_bits(peat_gpu.peat_product_f4(h, held[0], ops[1], None, 0, axes[1], None, dt(t)), want)
        assert same_bits(peat_gpu.peat_product_f4(h, ops[0], held[1], None, axes[0], 0, None, dt(t)), want)


@pytest.mark.parametrize("format", FORMATS)
def test_product_passes_bad_values_on(peat_gpu, h, format):
    """NaN and infinities make their row of the operand NaN."""
    import torch
    for M, K in ((5, 100), (300, 200), (300, 2000)):
        x = torch.randn(M, K, generator=rng(1), device="cuda").to(torch.bfloat16)
        w = torch.randn(260, K, generator=rng(2), device="cuda").to(torch.bfloat16)
        x[M // 2, K - 1] = float("inf")
        w[77, 0] = float("nan")
        for axis in (0, 1):
            u, v = (x, w) if axis == 0 else (x.t().contiguous(), w.t().contiguous())
            y = torch.isnan(peat_gpu.peat_product_f4(h, u, v, format, axis, axis))
            assert bool(y[M // 2].all()) and bool(y[:, 77].all()) and int(y.sum()) == M + 260 - 1


def test_product_refusals(peat_gpu, h):
    import torch
    P, x = peat_gpu, torch.randn(4, 64, device="cuda")
    m, n = P.peat_quantize_f4(h, x, "mxfp4"), P.peat_quantize_f4(h, x, "nvfp4")
    short = P.peat_quantize_f4(h, x[:, :32], "mxfp4")
    out = torch.empty(4, 4, device="cuda")
    for call in (lambda: P.peat_matmul_f4(h, m, n), lambda: P.peat_matmul_f4(h, m, short),
                 lambda: P.peat_matmul_f4_raw(h, m, m, out[:, :3]), lambda: P.peat_matmul_f4(h, m, m, x[0]),
                 lambda: P.peat_product_f4(h, x, x), lambda: P.peat_product_f4(h, m, x, "nvfp4"),
                 lambda: P.peat_product_f4(h, m, x, None, 1), lambda: P.peat_product_f4(h, m, x[:, :31]),
                 lambda: P.peat_product_f4(h, x, x[:, :63], "mxfp4"), lambda: P.peat_product_f4(h, x, x, "int4"),
                 lambda: P.Float4("mxfp4", m.q, m.block_scale[:-1]), lambda: P.Float4("mxfp4", m.q[:, :20], m.block_scale),
                 lambda: P.Float4("mxfp4", m.q, m.block_scale, n.scale), lambda: P.Float4("nvfp4", n.q, n.block_scale, n.scale[:3]),
                 lambda: P.Linear4(h, x, "mxfp8")):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        P.peat_matmul_f4(h, m, m, None, torch.float64)
    # rows off the 16-byte grid
    q = torch.zeros(4, 40, dtype=torch.uint8, device="cuda")[:, :32]
    with pytest.raises(P.PeatError) as e:
        P.peat_matmul_f4(h, P.Float4("mxfp4", q, m.block_scale), m)
    assert e.value.status == 1
    torch.cuda.synchronize()


@pytest.mark.parametrize("mnk", [(700, 300, 1024), (16, 700, 512), (16, 500, 8192), (300, 500, 16384), (4096, 4096, 512)])
def test_expired_wait_is_reported(peat_gpu, h, mnk):
    """A handle whose bounded waits give up at once: the product returns, the next one reports it, and other handles go
    on; tiles of a CTA, of few rows, of clusters that share k, of a pair."""
    import torch
    g = rng(3)
    M, N, K = mnk
    a, b = random_f4(peat_gpu, M, K, "nvfp4", g), random_f4(peat_gpu, N, K, "nvfp4", g)
    out = torch.empty(M, N, device="cuda")
    bad = peat_gpu.Handle(0, flags=peat_gpu.PEAT_FLAG_TEST_EXPIRE_WAITS)
    for _ in range(2):
        peat_gpu.peat_matmul_f4_raw(bad, a, b, out)
        torch.cuda.synchronize()
        with pytest.raises(peat_gpu.PeatError) as e:
            peat_gpu.peat_matmul_f4_raw(bad, a, b, out)
        assert e.value.status == 5
    bad.close()
    peat_gpu.peat_matmul_f4_raw(h, a, b, out)
    check_product(out, values64(a), values64(b), K, "nvfp4")


# tiles by pairs, clusters of two, four and eight that share k, with rows and columns that end inside a tile, and sums
# that the accumulators' shared columns, several waves and odd tiles go through
WAYS = [(4096, 4096, 512), (5000, 3001, 96), (2049, 8200, 1056), (16384, 300, 64), (1, 4096, 8192), (16, 4095, 4128),
        (48, 1000, 8192), (130, 500, 16384), (192, 512, 16384), (500, 520, 8192), (200, 300, 4096), (3, 100, 32768),
        (33, 9000, 4096), (17, 130, 520 * 32)]


@pytest.mark.parametrize("format", FORMATS)
@pytest.mark.parametrize("mnk", WAYS)
def test_matmul_ways(peat_gpu, h, format, mnk):
    import torch
    M, N, K = mnk
    g = rng(M + 3 * N + 7 * K)
    a, b = random_f4(peat_gpu, M, K, format, g), random_f4(peat_gpu, N, K, format, g)
    x, y = values64(a), values64(b)
    bias = torch.randn(N, generator=g, device="cuda") * K ** 0.5
    for bv, out, ldo in ((bias, torch.float32, N), (None, torch.bfloat16, (N + 7) // 8 * 8), (bias, torch.bfloat16, N + 1)):
        buf = torch.full((M, ldo), 7.0, device="cuda", dtype=out)
        peat_gpu.peat_matmul_f4_raw(h, a, b, buf[:, :N], bv)
        check_product(buf[:, :N], x, y, K, format, bv)
        assert bool((buf[:, N:] == 7).all())
        again = torch.empty(M, N, device="cuda", dtype=out)
        peat_gpu.peat_matmul_f4_raw(h, a, b, again, bv)
        if (ldo * again.element_size() % 16 == 0) == (N * again.element_size() % 16 == 0):
            assert same_bits(again, buf[:, :N])


@pytest.mark.parametrize("n", [1, 2, 3, 5, 9, 33])
def test_matmul_narrow_outputs(peat_gpu, h, n):
    """Fewer columns than a 16-byte unit, in rows on that grid."""
    import torch
    a, b = random_f4(peat_gpu, 300, 128, "mxfp4", rng(n)), random_f4(peat_gpu, n, 128, "mxfp4", rng(n + 1))
    for t in (torch.float32, torch.float16, torch.bfloat16):
        buf = torch.full((301, 40), 7.0, device="cuda", dtype=t)
        peat_gpu.peat_matmul_f4_raw(h, a, b, buf[:300, :n])
        if t != torch.float16 or float((values64(a) @ values64(b).t()).abs().max()) < 3e4:
            check_product(buf[:300, :n], values64(a), values64(b), 128, "mxfp4")
        assert bool((buf[:, n:] == 7).all()) and bool((buf[300:] == 7).all())


@pytest.mark.parametrize("format", FORMATS)
@pytest.mark.parametrize("m", [5, 300, 3000])
def test_matmul_scales_of_nan_and_zero(peat_gpu, h, format, m):
    """A block scale that is NaN makes its row NaN, one that is 0 (nvfp4) or the least (mxfp4) adds nothing."""
    import torch
    g = rng(m)
    a, b = random_f4(peat_gpu, m, 512, format, g), random_f4(peat_gpu, 260, 512, format, g)
    at = lambda r, k: ((r // 128) * (a.cols // BLOCK[format] // 4) + k // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + k % 4
    nan = 255 if format == "mxfp4" else 127
    a.block_scale[at(m - 1, 3)] = nan
    b.block_scale[at(200, 1)] = nan
    a.block_scale[at(1, 0)] = 0
    y = peat_gpu.peat_matmul_f4(h, a, b)
    bad = torch.isnan(y)
    assert bool(bad[m - 1].all()) and bool(bad[:, 200].all()) and int(bad.sum()) == m + 260 - 1
    # (a copy without the NaN, for the rest)
    a.block_scale[at(m - 1, 3)] = 127 if format == "mxfp4" else 56
    b.block_scale[at(200, 1)] = 127 if format == "mxfp4" else 56
    z = peat_gpu.peat_matmul_f4(h, a, b)
    check_product(z, values64(a), values64(b), 512, format)
    assert same_bits(z[: m - 1, :200], y[: m - 1, :200])


def test_small_and_large_scales(peat_gpu, h):
    """mxfp4's powers of two over float32's range: sums come out where they fit it, far apart ones too."""
    import torch
    for M in (4, 300):
        a, b = random_f4(peat_gpu, M, 128, "mxfp4", rng(1), 0), random_f4(peat_gpu, 40, 128, "mxfp4", rng(2), 0)
        for ea, eb in ((-120, 100), (110, -125), (-60, -60), (55, 60), (-100, 0)):
            a.block_scale.copy_(torch.where(a.block_scale > 0, 127 + ea, 0))
            b.block_scale.copy_(torch.where(b.block_scale > 0, 127 + eb, 0))
            check_product(peat_gpu.peat_matmul_f4(h, a, b), values64(a), values64(b), 128, "mxfp4")


# ---------------------------------------------------------------------------
# the layer
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("format", FORMATS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_linear4(peat_gpu, h, format, dtype):
    """Forward, input gradient and weight gradient of the rounded operands; leading dimensions, transposed inputs, a
    stream of its own."""
    import torch
    g = rng(9)
    x = torch.randn(3, 50, 200, generator=g, device="cuda").to(dt(dtype))
    w = (torch.randn(131, 200, generator=g, device="cuda") / 14).to(dt(dtype))
    grad = torch.randn(3, 50, 131, generator=g, device="cuda").to(dt(dtype))
    bias = torch.randn(131, generator=g, device="cuda")

    def val(t, axis):
        return definition(t, format, axis)[3].double()
    layer = peat_gpu.Linear4(h, w, format)
    rows, cols = x.reshape(-1, 200), grad.reshape(-1, 131)
    y = layer.forward(x, bias)
    assert y.shape == (3, 50, 131) and y.dtype == x.dtype
    check_product(y.view(-1, 131), val(rows, 0), val(w, 0), 224, format, bias)
    dx, dw = layer.backward(grad, x)
    check_product(dx.view(-1, 200), val(cols, 0), val(w, 1).t(), 160, format)
    assert dw.dtype == torch.float32
    check_product(dw, val(cols, 1).t(), val(rows, 1).t(), 160, format)
    assert same_bits(layer.forward(x.transpose(0, 1).contiguous().transpose(0, 1), bias), y)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = layer.forward(x, bias, stream=s), *layer.backward(grad, x, stream=s)
    s.synchronize()
    for a, b in zip(got, (y, dx, dw)):
        assert same_bits(a, b)
    none = layer.forward(x[:0])
    assert none.shape == (0, 50, 131)
    assert not bool(layer.weight_grad(grad[:0], x[:0]).any())


# ---------------------------------------------------------------------------
# norm
# ---------------------------------------------------------------------------
def norm_definition(x, residual, weight, eps):
    """(s, rstd, y float32, q, scale, values float32, rows whose mean of squares is not near a border)."""
    import torch
    s = x if residual is None else (x.double() + residual.double()).float().to(x.dtype)
    v64 = s.double().square().sum(1) / s.shape[1]
    v = v64.float()
    steps = [torch.nextafter(v, torch.full_like(v, d)) for d in (float("inf"), float("-inf"))]
    gap = torch.stack([((v.double() + t.double()) / 2 - v64).abs() for t in steps]).amin(0)
    # (on the border itself: 16-bit squares add up to few bits, exactly on both sides, and the even number is taken)
    clear = (gap > v64 * 2.0 ** -38) | (gap == 0) | ~torch.isfinite(v64) | (v64 == 0)
    e = torch.tensor(eps, dtype=torch.float32, device=x.device)
    rstd = (1.0 / single(torch.sqrt(single(v.double() + e.double())))).float()
    y = single(single(s.double() * rstd.double()[:, None]) * weight.double())
    bad = ~torch.isfinite(y).all(1)
    amax = torch.where(bad[:, None], 0.0, y).abs().amax(1)
    r = (127.0 / amax).float()
    zero = ~torch.isfinite(r) | bad
    r = torch.where(zero, 0.0, r)
    scale = torch.where(bad, float("nan"), torch.where(zero, 0.0, (amax / 127.0).float()))
    q = torch.round(single(torch.where(bad[:, None], 0.0, y) * r.double()[:, None])).to(torch.int8)
    return s, rstd, y.float(), q, scale, (q.double() * scale.double()[:, None]).float(), clear


def check_norm(P, h, x, residual, weight, eps=1e-6, pads=(0, 0, 0, 0), stream=None, most_unclear=0):
    import torch
    rows, cols = x.shape
    buf = [torch.full((rows + 1, cols + p), 7.0, dtype=x.dtype, device="cuda") for p in pads[:3]]
    s, y, v = (b[:rows, :cols] for b in buf)
    qbuf = torch.full((rows + 1, cols + pads[3]), 99, dtype=torch.int8, device="cuda")
    q = qbuf[:rows, :cols]
    scale, rstd = torch.full((rows,), -1.0, device="cuda"), torch.full((rows,), -1.0, device="cuda")
    P.peat_rmsnorm_raw(h, x, weight, eps, residual, s, y, q, scale, v, rstd, stream)
    torch.cuda.synchronize()
    es, er, ey, eq, esc, ev, clear = norm_definition(x, residual, weight, eps)
    assert int((~clear).sum()) <= most_unclear
    assert same_bits(s, es)
    assert same_bits(rstd[clear], er[clear])
    assert same_values(y[clear], ey.to(x.dtype)[clear])
    assert same_bits(scale[clear], esc[clear]) and torch.equal(q[clear], eq[clear])
    assert same_values(v[clear], ev.to(x.dtype)[clear])
    for b in buf:
        assert bool((b[rows:] == 7).all()) and bool((b[:, cols:] == 7).all())
    assert bool((qbuf[rows:] == 99).all()) and bool((qbuf[:, cols:] == 99).all())
    # each output alone gives the same
    y2, v2, q2 = torch.empty_like(es), torch.empty_like(es), torch.empty(rows, cols, dtype=torch.int8, device="cuda")
    r2, s2 = torch.empty_like(rstd), torch.empty_like(scale)
    P.peat_rmsnorm_raw(h, x, weight, eps, residual, y=y2, stream=stream)
    P.peat_rmsnorm_raw(h, x, weight, eps, residual, values=v2, stream=stream)
    P.peat_rmsnorm_raw(h, x, weight, eps, residual, q=q2, stream=stream)
    P.peat_rmsnorm_raw(h, x, weight, eps, residual, rstd=r2, stream=stream)
    P.peat_rmsnorm_raw(h, x, weight, eps, residual, scale=s2, stream=stream)
    torch.cuda.synchronize()
    assert same_values(y2, y) and same_values(v2, v) and torch.equal(q2, q) and same_bits(r2, rstd) and same_bits(s2, scale)


NORMS = [(1, 1), (1, 1024), (3, 17), (77, 1001), (64, 64), (9, 2056), (7, 4096), (5, 8192), (2, 16384), (3, 20000), (1000, 129),
         (4099, 40), (130, 257), (2, 70001)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", NORMS)
@pytest.mark.parametrize("add", [False, True])
def test_rmsnorm(peat_gpu, h, dtype, shape, add):
    import torch
    rows, cols = shape
    g = rng(rows * 7 + cols)
    for pad, off, pads, wt in ((0, 0, (0, 0, 0, 0), "f32"), (8, 0, (8, 16, 8, 16), dtype), (3, 1, (1, 3, 2, 5), "f32")):
        def make(scale):
            buf = (torch.randn(rows * (cols + pad) + off, generator=g, device="cuda") * scale).to(dt(dtype))
            return buf[off:].view(rows, cols + pad)[:, :cols]
        x, r = make(2.0), make(5.0) if add else None
        w = (1 + 0.3 * torch.randn(cols, generator=g, device="cuda")).to(dt(wt))
        check_norm(peat_gpu, h, x, r, w, pads=pads, most_unclear=rows // 1000)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [40, 1000, 3000, 20000])
def test_rmsnorm_extremes(peat_gpu, h, dtype, cols):
    """Rows of zeros, of the type's largest and smallest numbers, NaN and infinities; without eps too."""
    import torch
    big, tiny = torch.finfo(dt(dtype)).max, torch.finfo(dt(dtype)).smallest_normal
    x = torch.randn(10, cols, generator=rng(cols), device="cuda")
    x[0] = 0.0
    x[1] = torch.where(x[1] > 0, big, -big)
    x[2] = torch.where(x[2] > 0, tiny, -tiny)
    x[3] = 0.0
    x[3, cols - 1] = tiny
    x[4, 0] = float("nan")
    x[5, cols // 2] = float("inf")
    x[6] *= 2.0 ** -30 if dtype != "f16" else 2.0 ** -12
    x[7, 1] = big
    w = 1 + 0.1 * torch.randn(cols, generator=rng(1), device="cuda")
    for eps in (1e-6, 1e-30, 0.0):
        check_norm(peat_gpu, h, x.to(dt(dtype)), None, w, eps)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols,pad", [(64, 0), (1000, 0), (1001, 0), (4096, 3), (20000, 1)])
def test_rmsnorm_in_place(peat_gpu, h, dtype, cols, pad):
    """The sum takes the place of x, or of the residual."""
    import torch
    g = rng(cols)
    make = lambda: torch.randn(33, cols + pad, generator=g, device="cuda").to(dt(dtype))[:, :cols]
    x, r, w = make(), make(), torch.randn(cols, generator=g, device="cuda")
    es, er, ey, eq, esc, ev, clear = norm_definition(x, r, w, 1e-5)
    assert bool(clear.all())
    for which in (0, 1):
        bufs = [x.clone(), r.clone()]
        y, q = torch.empty(33, cols, dtype=x.dtype, device="cuda"), torch.empty(33, cols, dtype=torch.int8, device="cuda")
        peat_gpu.peat_rmsnorm_raw(h, bufs[0], w, 1e-5, bufs[1], sum=bufs[which], y=y, q=q)
        assert same_bits(bufs[which], es) and same_bits(bufs[1 - which], (r, x)[which])
        assert same_values(y, ey.to(x.dtype)) and torch.equal(q, eq)


def backward_definition(grad, x, weight, rstd, stream):
    import torch
    r, d, w = rstd.double()[:, None], grad.double(), weight.double()
    n = x.double() * r
    g = d * w
    c = (g * n).mean(1, keepdim=True) if x.shape[1] else 0.0
    dx = r * (g - n * c)
    cols = x.shape[1]
    ctol = ((32 + cols / 256 + 20 + 3) * EPS) * (g * n).abs().mean(1, keepdim=True)
    tol = r.abs() * (n.abs() * ctol + 5 * EPS * (g.abs() + (n * c).abs())) + EPS * dx.abs()
    if stream is not None:
        dx = dx + stream.double()
        tol = tol + EPS * dx.abs()
    rows = x.shape[0]
    wsum = (d * n).abs().sum(0)
    return dx, tol, (d * n).sum(0), (rows / 400 + 64 + 4) * EPS * wsum


def check_backward(P, h, grad, x, weight, rstd, add, pad=0, stream=None):
    import torch
    rows, cols = x.shape
    buf = torch.full((rows + 1, cols + pad), 7.0, dtype=x.dtype, device="cuda")
    dx, dw = buf[:rows, :cols], torch.full((cols,), 7.0, device="cuda")
    P.peat_rmsnorm_backward_raw(h, grad, x, weight, rstd, dx, dw, add, stream)
    torch.cuda.synchronize()
    ex, tol, ew, wtol = backward_definition(grad, x, weight, rstd, add)
    if x.dtype != torch.float32:
        fi = torch.finfo(x.dtype)
        tol = tol + (ex.abs() + tol) * fi.eps / 2 + fi.smallest_normal * fi.eps / 2
    assert bool(((dx.double() - ex).abs() <= tol).all()), float(((dx.double() - ex).abs() / tol.clamp(min=1e-300)).max())
    assert bool(((dw.double() - ew).abs() <= wtol).all()), float(((dw.double() - ew).abs() / wtol.clamp(min=1e-300)).max())
    assert bool((buf[rows:] == 7).all()) and bool((buf[:, cols:] == 7).all())
    # each output alone gives the same
    dx2, dw2 = torch.empty(rows, cols, dtype=x.dtype, device="cuda"), torch.empty(cols, device="cuda")
    P.peat_rmsnorm_backward_raw(h, grad, x, weight, rstd, dx2, None, add, stream)
    P.peat_rmsnorm_backward_raw(h, grad, x, weight, rstd, None, dw2, add, stream)
    torch.cuda.synchronize()
    assert same_bits(dx2, dx) and same_bits(dw2, dw)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", NORMS + [(0, 40), (5000, 1000), (700, 2000)])
@pytest.mark.parametrize("add", [False, True])
def test_rmsnorm_backward(peat_gpu, h, dtype, shape, add):
    import torch
    rows, cols = shape
    g = rng(rows * 5 + cols)
    for pad, off, opad, wt in ((0, 0, 0, "f32"), (8, 0, 8, dtype), (3, 1, 1, "f32")):
        def make(scale):
            buf = (torch.randn(rows * (cols + pad) + off, generator=g, device="cuda") * scale).to(dt(dtype))
            return buf[off:].view(rows, cols + pad)[:, :cols]
        x, grad, r = make(2.0), make(0.1), make(0.2) if add else None
        w = (1 + 0.3 * torch.randn(cols, generator=g, device="cuda")).to(dt(wt))
        rstd = (1.0 / torch.sqrt(x.double().square().mean(1) + 1e-6)).float()
        check_backward(peat_gpu, h, grad, x, w, rstd, r, opad)


@pytest.mark.parametrize("cols,pad", [(64, 0), (1001, 0), (4096, 3), (20000, 1)])
def test_rmsnorm_backward_in_place(peat_gpu, h, cols, pad):
    """The gradient takes the place of grad, or of the stream's."""
    import torch
    g = rng(cols)
    make = lambda: torch.randn(333, cols + pad, generator=g, device="cuda").to(torch.bfloat16)[:, :cols]
    x, grad, r, w = make(), make(), make(), torch.randn(cols, generator=g, device="cuda")
    rstd = torch.rand(333, generator=g, device="cuda") + 0.5
    want, dw = peat_gpu.peat_rmsnorm_backward(h, grad, x, w, rstd, r)
    for which in (0, 1):
        bufs = [grad.clone(), r.clone()]
        got = torch.empty(cols, device="cuda")
        peat_gpu.peat_rmsnorm_backward_raw(h, bufs[0], x, w, rstd, bufs[which], got, bufs[1])
        assert same_bits(bufs[which], want) and same_bits(got, dw) and same_bits(bufs[1 - which], (r, grad)[which])


def test_rmsnorm_backward_against_differences(peat_gpu, h):
    """The gradients are those of the norm: central differences of its 64-bit form."""
    import torch
    g = rng(4)
    x, w = torch.randn(3, 24, generator=g, device="cuda"), 1 + 0.3 * torch.randn(24, generator=g, device="cuda")
    d, up = torch.randn(3, 24, generator=g, device="cuda"), torch.randn(3, 24, generator=g, device="cuda")

    def loss(xv, wv):  # of y and of the stream itself
        r = 1.0 / torch.sqrt(xv.square().mean(1, keepdim=True) + 1e-6)
        return float(((xv * r * wv) * d.double()).sum() + (xv * up.double()).sum())
    got = peat_gpu.peat_rmsnorm(h, x, w, 1e-6)
    dx, dw = peat_gpu.peat_rmsnorm_backward(h, d, x, w, got["rstd"], up)
    step = 1e-5  # differences are off by step^2 times third derivatives, and by 1e-16 / step of the loss
    for i in range(3):
        for j in range(24):
            e = torch.zeros(3, 24, dtype=torch.float64, device="cuda")
            e[i, j] = step
            fd = (loss(x.double() + e, w.double()) - loss(x.double() - e, w.double())) / (2 * step)
            assert abs(fd - float(dx[i, j])) <= 1e-5 * (1 + abs(fd))
    for j in range(24):
        e = torch.zeros(24, dtype=torch.float64, device="cuda")
        e[j] = step
        fd = (loss(x.double(), w.double() + e) - loss(x.double(), w.double() - e)) / (2 * step)
        assert abs(fd - float(dw[j])) <= 1e-5 * (1 + abs(fd))


def test_rmsnorm_refusals(peat_gpu, h):
    import torch
    P, x, w = peat_gpu, torch.zeros(4, 8, device="cuda"), torch.ones(8, device="cuda")
    v, q = torch.zeros(4, device="cuda"), torch.zeros(4, 8, dtype=torch.int8, device="cuda")
    for call in (lambda: P.peat_rmsnorm_raw(h, x, w[:7], y=x), lambda: P.peat_rmsnorm_raw(h, x, w, residual=x[:, :7], y=x),
                 lambda: P.peat_rmsnorm_raw(h, x, w, y=x.half()), lambda: P.peat_rmsnorm_raw(h, x, w, q=x),
                 lambda: P.peat_rmsnorm_raw(h, x, w, rstd=v[:3]), lambda: P.peat_rmsnorm_raw(h, x.t(), w, y=x),
                 lambda: P.peat_rmsnorm_raw(h, x, torch.ones(8), y=x), lambda: P.peat_rmsnorm(h, x[0], w),
                 lambda: P.peat_rmsnorm_backward_raw(h, x, x, w, None, x), lambda: P.peat_rmsnorm_backward_raw(h, x, x, w, v[:2], x),
                 lambda: P.peat_rmsnorm_backward_raw(h, x[:3], x, w, v, x), lambda: P.RMSNorm8(h, w).forward(x[:, :4])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        P.peat_rmsnorm_raw(h, x, w.half(), y=x)
    for call in (lambda: P.peat_rmsnorm_raw(h, x, w), lambda: P.peat_rmsnorm_raw(h, x, w, -1.0, y=q.float()),
                 lambda: P.peat_rmsnorm_raw(h, x, w, float("nan"), y=q.float()), lambda: P.peat_rmsnorm_backward_raw(h, x, x, w, v)):
        with pytest.raises(P.PeatError) as e:
            call()
        assert e.value.status == 1


# ---------------------------------------------------------------------------
# together, on streams, in graphs
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sublayer(peat_gpu, h, dtype):
    """A sublayer as it is replayed: norm to 8 bits, 8-bit product; norm, 4-bit product; the gradients back through both."""
    import torch
    g = rng(12)
    x, r = (torch.randn(2, 65, 200, generator=g, device="cuda").to(dt(dtype)) for _ in range(2))
    wn = 1 + 0.2 * torch.randn(200, generator=g, device="cuda")
    w = (torch.randn(300, 200, generator=g, device="cuda") / 14).to(dt(dtype))
    norm, layer = peat_gpu.RMSNorm8(h, wn), peat_gpu.Linear8(h, w)
    got = norm.forward(x, r)
    assert got["q"].shape == x.shape and got["scale"].shape == (2, 65)
    s, rstd, y, q, scale, values, clear = norm_definition(x.view(-1, 200), r.view(-1, 200), wn, 1e-6)
    assert bool(clear.all()) and torch.equal(got["q"].view(-1, 200), q) and same_bits(got["sum"].view(-1, 200), s)
    out = layer.forward_rounded(got["q"], got["scale"], dt(dtype))
    wq, ws = peat_gpu.peat_quantize_i8(h, w, 0)
    want = (q.double() @ wq.double().t()).float() * (scale[:, None] * ws[None, :])
    assert out.shape == (2, 65, 300) and same_bits(out.view(-1, 300), want.to(dt(dtype)))
    # the 4-bit layer takes the norm's output as it is
    plain = peat_gpu.peat_rmsnorm(h, x.view(-1, 200), wn, residual=r.view(-1, 200), rounded=False)
    for format in FORMATS:
        z = peat_gpu.Linear4(h, w, format).forward(plain["y"])
        check_product(z, definition(plain["y"], format, 0)[3].double(), definition(w, format, 0)[3].double(), 224, format)
    # and back
    up = torch.randn(2, 65, 300, generator=g, device="cuda").to(dt(dtype))
    dy = layer.input_grad(up)
    dx, dw = norm.backward(dy, got["sum"], got["rstd"], r)
    ex, tol, ew, wtol = backward_definition(dy.view(-1, 200), s, wn, rstd, r.view(-1, 200))
    if dtype != "f32":
        tol = tol + (ex.abs() + tol) * torch.finfo(dt(dtype)).eps / 2
    assert dx.shape == x.shape and bool(((dx.view(-1, 200).double() - ex).abs() <= tol).all())
    assert bool(((dw.double() - ew).abs() <= wtol).all())


def test_streams(peat_gpu, h):
    """Calls on a stream of their own, behind work that is slow on it."""
    import torch
    P, g = peat_gpu, rng(8)
    x, w = torch.randn(300, 500, generator=g, device="cuda"), torch.randn(200, 500, generator=g, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        y = x * 2
    a = P.peat_quantize_f4(h, y, "nvfp4", stream=s)
    b = P.peat_quantize_f4(h, w, "nvfp4", stream=s)
    z = P.peat_matmul_f4(h, a, b, stream=s)
    n = P.peat_rmsnorm(h, y, torch.ones(500, device="cuda"), stream=s)
    s.synchronize()
    check_product(z, definition(x * 2, "nvfp4", 0)[3].double(), definition(w, "nvfp4", 0)[3].double(), 512, "nvfp4")
    assert torch.equal(n["q"], norm_definition(x * 2, None, torch.ones(500, device="cuda"), 1e-6)[3])


def test_captured_calls(peat_gpu):
    """Calls captured into a graph and replayed on new inputs, between calls that are not, and after the workspace has
    grown."""
    import torch
    P, g = peat_gpu, rng(21)
    with P.Handle(0) as h:
        x, w = torch.empty(300, 500, device="cuda"), torch.empty(260, 500, device="cuda")
        wn, grad = torch.empty(500, device="cuda"), torch.empty(300, 500, device="cuda")
        y = {f: torch.empty(300, 260, device="cuda") for f in FORMATS}
        yt = torch.empty(500, 500, device="cuda")
        q, sc, rs = torch.empty(300, 500, dtype=torch.int8, device="cuda"), torch.empty(300, device="cuda"), torch.empty(300, device="cuda")
        dx, dw = torch.empty(300, 500, device="cuda"), torch.empty(500, device="cuda")

        def fill():
            for t in (x, w, grad, wn):
                t.copy_(torch.randn(t.shape, generator=g, device="cuda"))

        def calls():
            for f in FORMATS:
                P.peat_product_f4_raw(h, x, w, y[f], f)
            P.peat_product_f4_raw(h, x, grad, yt, "nvfp4", 1, 1)
            P.peat_rmsnorm_raw(h, x, wn, q=q, scale=sc, rstd=rs)
            P.peat_rmsnorm_backward_raw(h, grad, x, wn, rs, dx, dw)

        def check():
            torch.cuda.synchronize()
            for f in FORMATS:
                check_product(y[f], definition(x, f, 0)[3].double(), definition(w, f, 0)[3].double(), 512, f)
            check_product(yt, definition(x, "nvfp4", 1)[3].double().t(), definition(grad, "nvfp4", 1)[3].double().t(), 304, "nvfp4")
            s, rstd, _, eq, esc, _, clear = norm_definition(x, None, wn, 1e-6)
            assert torch.equal(q[clear], eq[clear]) and int((~clear).sum()) == 0
            ex, tol, ew, wtol = backward_definition(grad, x, wn, rstd, None)
            assert bool(((dx.double() - ex).abs() <= tol).all()) and bool(((dw.double() - ew).abs() <= wtol).all())
        fill()
        calls()
        check()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls()
        for turn in range(3):
            fill()
            for t in (*y.values(), yt, q, sc, rs, dx, dw):
                t.zero_()
            graph.replay()
            check()
            calls()
            check()
            big = torch.randn(900 * (turn + 1), 2000, generator=g, device="cuda")
            P.peat_product_f4(h, big, big, "nvfp4", 1, 1)
            P.peat_rmsnorm_backward(h, big, big, torch.ones(2000, device="cuda"), torch.ones(big.shape[0], device="cuda"))


def test_capture_that_would_allocate_is_refused(peat_gpu):
    import torch
    P = peat_gpu
    x = torch.randn(64, 64, device="cuda")
    out = torch.empty(64, 64, device="cuda")
    with P.Handle(0) as h:
        g = torch.cuda.CUDAGraph()
        with pytest.raises(P.PeatError) as e:
            with torch.cuda.graph(g):
                P.peat_product_f4_raw(h, x, x, out, "mxfp4")
        assert e.value.status == 2
        P.peat_product_f4_raw(h, x, x, out, "mxfp4")
        torch.cuda.synchronize()


def test_rows_past_32_bit_offsets(peat_gpu, h):
    """A matrix of more than 2^32 bytes, its last rows."""
    import torch
    rows, cols = 40000, 65536
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(200, cols, generator=rng(2), device="cuda").to(torch.bfloat16)
    x[-200:] = tail
    w = torch.randn(32, cols, generator=rng(3), device="cuda").to(torch.bfloat16)
    for format in FORMATS:
        a, b = peat_gpu.peat_quantize_f4(h, x, format), peat_gpu.peat_quantize_f4(h, w, format)
        t = peat_gpu.peat_quantize_f4(h, tail, format)
        assert torch.equal(a.q[-200:], t.q)
        y = peat_gpu.peat_matmul_f4(h, a, b)
        # (against the 64-bit product: a call of other sizes may add in another order)
        check_product(y[-200:], values64(t), values64(b), cols, format)
        assert not bool(y[:-200].any())
        del a, y
    one = torch.ones(cols, device="cuda")
    got = peat_gpu.peat_rmsnorm(h, x, one)
    assert torch.equal(got["q"][-200:], peat_gpu.peat_rmsnorm(h, tail, one)["q"])
    dx, dw = peat_gpu.peat_rmsnorm_backward(h, x, x, one, got["rstd"])
    ex, ew = peat_gpu.peat_rmsnorm_backward(h, tail, tail, one, got["rstd"][-200:].contiguous())
    assert same_bits(dx[-200:], ex) and not bool(dx[:-200].any())
    assert float((dw - ew).abs().max()) <= 300 * EPS * float((tail.double().square().sum(0) * got["rstd"][-200:].max().double()).max())


def test_another_current_device_and_default_stream(peat_gpu):
    """A handle's calls run on its device whatever else is current (one GPU: device 0 by number)."""
    import torch
    with peat_gpu.Handle(0) as h:
        x = torch.randn(40, 64, device="cuda:0")
        got = peat_gpu.peat_quantize_f4(h, x, "mxfp4")
        assert same_values(got.values(), definition(x, "mxfp4", 0)[3])
        assert np.isfinite(float(peat_gpu.peat_rmsnorm(h, x, torch.ones(64, device="cuda"))["rstd"].sum()))
