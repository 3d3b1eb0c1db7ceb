"""The playback operators (quantisation, 8-bit products, gradient norm and
clipping, the 8-bit linear layer) against their definitions in 64 bits.

Tolerances.  Integers, scales, values, products and clipped elements are
defined by single float32 roundings that binary64 reproduces (a product of two
float32 values is exact in binary64, a quotient rounds to the same float32), so
they have to be equal.  A norm sums at most 64 elements in plain float32, each
step off by 2^-24 of the sum, and the rest with the error kept: 64 2^-24 on the
sum of squares, half of that on its root, 2^-24 for the result: 40 2^-24 covers
the 2-norm, 70 2^-24 the 1-norm.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
TOL = {"2": 40 * EPS, "1": 70 * EPS, "inf": EPS}


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


# ---------------------------------------------------------------------------
# quantisation
# ---------------------------------------------------------------------------
def quant_definition(x, axis):
    """(q int8, scale float32, values of x's type), from binary64, by row of x (axis 0) or of its transpose."""
    import torch
    v = x.double().t() if axis else x.double()
    n = v.shape[1]
    amax = v.abs().amax(1) if n else torch.zeros(v.shape[0], dtype=torch.float64, device=x.device)
    bad = ~torch.isfinite(v).all(1) if n else torch.zeros_like(amax, dtype=torch.bool)
    r = (127.0 / amax).float()
    zero = ~torch.isfinite(r) | bad
    r = torch.where(zero, torch.zeros_like(r), r)
    scale = torch.where(zero, torch.zeros_like(r), (amax / 127.0).float())
    scale = torch.where(bad, torch.full_like(scale, float("nan")), scale)
    vv = torch.where(bad[:, None], torch.zeros_like(v), v)
    q = torch.round((vv * r.double()[:, None]).float().double()).to(torch.int8)
    val = (q.double() * scale.double()[:, None]).float().to(x.dtype)
    return q, scale, (val.t() if axis else val)


def check_quant(peat, h, x, axis, qpad=0, vpad=0, stream=None):
    import torch
    rows, cols = x.shape
    qr, qc = (cols, rows) if axis else (rows, cols)
    qbuf = torch.full((qr + 1, qc + qpad), 99, dtype=torch.int8, device="cuda")
    vbuf = torch.full((rows + 1, cols + vpad), 7.0, dtype=x.dtype, device="cuda")
    q, v = qbuf[:qr, :qc], vbuf[:rows, :cols]
    scale = torch.full((qr,), -1.0, device="cuda")
    peat.peat_quantize_i8_raw(h, x, axis, q, scale, v, stream)
    torch.cuda.synchronize()
    eq, es, ev = quant_definition(x, axis)
    assert same_bits(scale, es)
    assert torch.equal(q, eq)
    assert same_bits(v, ev)
    assert bool((qbuf[qr:] == 99).all()) and bool((qbuf[:, qc:] == 99).all())
    assert bool((vbuf[rows:] == 7).all()) and bool((vbuf[:, cols:] == 7).all())
    # each output alone gives the same
    q2, v2 = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty_like(v, memory_format=torch.contiguous_format)
    peat.peat_quantize_i8_raw(h, x, axis, q2, None, None, stream)
    peat.peat_quantize_i8_raw(h, x, axis, None, None, v2, stream)
    torch.cuda.synchronize()
    assert torch.equal(q2, eq) and same_bits(v2, ev)


SHAPES = [(1, 1), (1, 1024), (3, 17), (5, 1000), (64, 64), (130, 257), (9, 2056), (7, 4096), (2, 16384), (3, 20000),
          (1000, 129), (4099, 40), (513, 72)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("shape", SHAPES)
def test_quantize(peat_gpu, h, dtype, axis, shape):
    import torch
    rows, cols = shape
    g = rng(rows * 31 + cols)
    for pad, off, qpad, vpad in ((0, 0, 0, 0), (8, 0, 16, 8), (3, 1, 5, 1)):
        buf = torch.randn(rows * (cols + pad) + off, generator=g, device="cuda").to(dt(dtype))
        x = buf[off:].view(rows, cols + pad)[:, :cols]
        check_quant(peat_gpu, h, x, axis, qpad, vpad)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("axis", [0, 1])
def test_quantize_extremes(peat_gpu, h, dtype, axis):
    """Rows of zeros, negative zeros, the type's largest and smallest values, ties, NaN and infinities."""
    import torch
    big, tiny = torch.finfo(dt(dtype)).max, torch.finfo(dt(dtype)).smallest_normal
    sub = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}[dtype]
    x = torch.randn(12, 300, generator=rng(1), device="cuda")
    x[0] = 0.0
    x[1] = -0.0
    x[2] = torch.where(x[2] > 0, big, -big)
    x[3] = x[3].sign() * tiny
    x[4] = x[4].sign() * sub
    x[5] = torch.arange(300, device="cuda") * 0.5 - 75.0
    x[5, 0] = 127.0  # r = 1: every half is a tie
    x[6, 17] = float("nan")
    x[7, 299] = float("inf")
    x[8, 0] = -float("inf")
    x[8, 1] = float("nan")
    x[9] = 0.0
    x[9, 250] = -big
    x[10] = big
    x[11] = 3e-37 if dtype != "f16" else 1e-7
    x = x.to(dt(dtype))
    check_quant(peat_gpu, h, x if axis == 0 else x.t().contiguous(), axis)


@pytest.mark.parametrize("axis", [0, 1])
def test_quantize_empty(peat_gpu, h, axis):
    import torch
    for rows, cols in ((0, 5), (5, 0), (0, 0)):
        x = torch.zeros(rows, cols, device="cuda")
        n = cols if axis else rows
        scale = torch.full((n,), -1.0, device="cuda")
        q = torch.empty((cols, rows) if axis else (rows, cols), dtype=torch.int8, device="cuda")
        peat_gpu.peat_quantize_i8_raw(h, x, axis, q, scale)
        assert scale.tolist() == [0.0] * n


# ---------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------
def ints(rows, cols, fill, g, pad=0, off=0):
    import torch
    buf = torch.full((rows * (cols + pad) + off + 16,), 77, dtype=torch.int8, device="cuda")
    x = buf[off : off + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    if fill == "uniform":
        x.copy_(torch.randint(-128, 128, (rows, cols), generator=g, device="cuda", dtype=torch.int8))
    elif fill == "gauss":
        x.copy_((torch.randn(rows, cols, generator=g, device="cuda") * 32).round().clamp(-127, 127))
    elif fill == "low":
        x.fill_(-128)
    else:  # one sign, large, not all even
        x.copy_(127 - (torch.rand(rows, cols, generator=g, device="cuda") < 0.3).to(torch.int8))
    return x


def sums(a, b):
    """The exact integer products: int64 through binary64 (below 2^53)."""
    import torch
    return (a.double() @ b.double().t()).round().to(torch.int64)


MNK = [(1, 1, 1), (1, 4096, 1024), (2, 50, 63), (8, 129, 64), (9, 16, 65), (16, 1000, 2049), (17, 33, 100),
       (5, 40, 16384), (33, 70, 513), (64, 128, 64), (65, 129, 640), (100, 300, 4097), (128, 256, 512),
       (257, 511, 1030), (300, 1000, 777), (128, 100, 9000), (1000, 1, 300), (1025, 769, 2080)]


@pytest.mark.parametrize("fill", ["uniform", "gauss", "low", "high"])
@pytest.mark.parametrize("mnk", MNK)
def test_matmul_sums(peat_gpu, h, fill, mnk):
    """The integer sums, exactly, up to their bound, from rows of any alignment."""
    import torch
    M, N, K = mnk
    g = rng(M + N + K)
    for pa, oa, pb, ob in ((-K % 16, 0, -K % 16, 0), (0, 0, 0, 0), (1, 3, 4, 0)):
        a, b = ints(M, K, fill, g, pa, oa), ints(N, K, fill, g, pb, ob)
        buf = torch.full((M + 1, N + 3), -5, dtype=torch.int32, device="cuda")
        peat_gpu.peat_matmul_i8_raw(h, a, None, b, None, buf[:M, :N])
        assert torch.equal(buf[:M, :N].to(torch.int64), sums(a, b)), (pa, oa)
        assert bool((buf[M:] == -5).all()) and bool((buf[:, N:] == -5).all())


@pytest.mark.parametrize("mnk", [(1, 7, 131071), (20, 40, 131071), (300, 300, 131071), (600, 520, 20000)])
@pytest.mark.parametrize("fill", ["low", "uniform"])
def test_matmul_long_sums(peat_gpu, h, fill, mnk):
    import torch
    M, N, K = mnk
    g = rng(K)
    a, b = ints(M, K, fill, g, -K % 16), ints(N, K, fill, g, -K % 16)
    out = torch.empty(M, N, dtype=torch.int32, device="cuda")
    peat_gpu.peat_matmul_i8_raw(h, a, None, b, None, out)
    assert torch.equal(out.to(torch.int64), sums(a, b))


@pytest.mark.parametrize("out", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("mnk", [(1, 4096, 1024), (16, 50257, 1024), (17, 31, 33), (257, 1000, 2049), (512, 1024, 1024),
                                 (640, 1111, 320), (2048, 1024, 4096)])
@pytest.mark.parametrize("bias", [False, True])
def test_matmul_scaled(peat_gpu, h, out, mnk, bias):
    """One rounding of the sum, one of the scales' product, one of each operation: float32 arithmetic reproduces it."""
    import torch
    M, N, K = mnk
    g = rng(M * 3 + N)
    a, b = ints(M, K, "gauss", g, -K % 16), ints(N, K, "gauss", g, -K % 16)
    sa = torch.rand(M, generator=g, device="cuda") * 0.1
    sb = torch.rand(N, generator=g, device="cuda") * 0.1
    bv = torch.randn(N, generator=g, device="cuda") if bias else None
    want = sums(a, b).float() * (sa[:, None] * sb[None, :])
    if bias:
        want = want + bv
    for pad in (0, 1, 8):
        buf = torch.full((M + 1, N + pad), 3.0, dtype=dt(out), device="cuda")
        peat_gpu.peat_matmul_i8_raw(h, a, sa, b, sb, buf[:M, :N], bv)
        assert same_bits(buf[:M, :N], want.to(dt(out)))
        assert bool((buf[M:] == 3).all()) and bool((buf[:, N:] == 3).all())
    got = peat_gpu.peat_matmul_i8(h, a, None, b, sb, out_dtype=dt(out))
    assert same_bits(got, (sums(a, b).float() * sb).to(dt(out)))


def test_matmul_edges(peat_gpu, h):
    """K = 0, no rows, NaN scales."""
    import torch
    z = torch.zeros(300, 0, dtype=torch.int8, device="cuda")
    bias = torch.arange(300, device="cuda", dtype=torch.float32)
    assert torch.equal(peat_gpu.peat_matmul_i8(h, z, None, z, None, bias), bias.expand(300, 300))
    e = torch.zeros(0, 8, dtype=torch.int8, device="cuda")
    assert peat_gpu.peat_matmul_i8(h, e, None, z[:, :0].new_zeros(5, 8), None).shape == (0, 5)
    for M in (1, 40, 700):
        a = torch.ones(M, 64, dtype=torch.int8, device="cuda")
        b = torch.ones(600, 64, dtype=torch.int8, device="cuda")
        sa = torch.ones(M, device="cuda")
        sa[M // 2] = float("nan")
        y = peat_gpu.peat_matmul_i8(h, a, sa, b, None)
        assert bool(torch.isnan(y[M // 2]).all()) and int(torch.isnan(y).sum()) == 600
        assert bool((y[torch.arange(M, device="cuda") != M // 2] == 64).all())


def test_matmul_repeats_and_sizes_in_turn(peat_gpu, h):
    """Calls of different sizes one after another on one handle, nothing waiting between them: the workspace of one
    is the next one's; the same call gives the same bits."""
    import torch
    g = rng(5)
    jobs = []
    for M, N, K in ((700, 900, 1100), (1, 64, 64), (2100, 520, 130), (700, 900, 1100), (260, 260, 5000)):
        a, b = ints(M, K, "uniform", g, -K % 16), ints(N, K, "uniform", g, -K % 16)
        jobs.append((a, b, torch.empty(M, N, dtype=torch.int32, device="cuda")))
    for _ in range(3):
        for a, b, o in jobs:
            o.fill_(-1)
        for a, b, o in jobs:
            peat_gpu.peat_matmul_i8_raw(h, a, None, b, None, o)
        for a, b, o in jobs:
            assert torch.equal(o.to(torch.int64), sums(a, b))


# ---------------------------------------------------------------------------
# gradient lists
# ---------------------------------------------------------------------------
def norm64(t, kind):
    import torch
    v = t.double().flatten()
    if v.numel() == 0:
        return 0.0
    return float(torch.linalg.vector_norm(v, {"2": 2, "1": 1, "inf": float("inf")}[kind]))


def check_list(peat, h, ts, kind="2", unscale=1.0, outs=None, max_norm=None, eps=1e-6, bad="propagate", stream=None):
    """Norms against 64 bits; the factor and every clipped element from the reported norm, exactly."""
    import torch
    before = [t.clone() for t in ts]
    want = [norm64(t, kind) * unscale for t in ts]
    total = {"2": lambda w: float(np.sqrt(np.sum(np.square(w)))), "1": lambda w: float(np.sum(w)),
             "inf": lambda w: float(np.max(w)) if len(w) else 0.0}[kind](np.array(want, np.float64))
    glist = peat.GradList(ts, outs)
    if max_norm is None:
        r = peat.peat_grad_norm(h, glist, kind, unscale, stream)
        assert r["coef"] == 1.0
    else:
        r = peat.peat_grad_clip(h, glist, max_norm, kind, unscale, eps, bad, stream)
    n_bad = sum(int((~torch.isfinite(t)).sum()) for t in before)
    assert r["n_bad"] == n_bad
    for got, w in list(zip(r["norms"].tolist(), want)) + [(r["norm"], total)]:
        if not np.isfinite(w):
            assert (np.isnan(w) and np.isnan(got)) or w == got, (got, w)
        else:
            assert abs(got - w) <= TOL[kind] * w + 2.0 ** -150, (got, w)
    if max_norm is not None:
        with np.errstate(all="ignore"):
            q = np.float32(max_norm) / (np.float32(r["norm"]) + np.float32(eps))
        c = np.float32(1.0) if q >= 1 else q
        if n_bad and bad != "propagate":
            c = np.float32(0.0 if bad == "zero" else 1.0)
        assert np.float32(r["coef"]).tobytes() == np.float32(c).tobytes() or (np.isnan(c) and np.isnan(r["coef"]))
        f = np.float32(unscale) * c
        for t, b, o in zip(ts, before, outs if outs is not None else ts):
            w = torch.zeros_like(b) if n_bad and bad == "zero" else (b.float() * float(f)).to(b.dtype)
            assert same_bits(o, w)
            if outs is not None and o is not t:
                assert same_bits(t, b)
    return r


def grads(sizes, dtypes, seed, scale=1.0, shift=0):
    import torch
    g = rng(seed)
    out = []
    for i, n in enumerate(sizes):
        d = dt(dtypes[i % len(dtypes)])
        out.append((torch.randn(n + shift, generator=g, device="cuda") * scale).to(d)[shift:])
    return out


LISTS = [[0], [1], [7], [64], [1000], [4099], [0, 0, 5, 0], [1, 2, 3, 4, 5, 6, 7, 8, 9], [100003, 0, 17, 65536, 1],
         [64] * 97, [33] * 400, [1 << 20, 3, (1 << 20) + 5], [0] * 5]


@pytest.mark.parametrize("kind", ["2", "1", "inf"])
@pytest.mark.parametrize("dtypes", [("f32",), ("f16",), ("bf16",), ("bf16", "f32", "f16")])
@pytest.mark.parametrize("which", range(len(LISTS)))
def test_grad_lists(peat_gpu, h, kind, dtypes, which):
    import torch
    for shift in (0, 1):
        ts = grads(LISTS[which], dtypes, which, 0.1, shift)
        check_list(peat_gpu, h, ts, kind)
        outs = [torch.full((t.numel() + 3,), 9.0, dtype=t.dtype, device="cuda") for t in ts]
        check_list(peat_gpu, h, ts, kind, 0.5, [o[:-3] for o in outs], 0.7)
        assert all(bool((o[-3:] == 9).all()) for o in outs)
        outs = [torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")[1:] for t in ts]  # off the input's grid, or not
        check_list(peat_gpu, h, ts, kind, 1.0, outs, 1e9)
        check_list(peat_gpu, h, ts, kind, 1.0, None, 0.3)  # in place


def test_empty_list(peat_gpu, h):
    r = peat_gpu.peat_grad_clip(h, [], 1.0)
    assert r["norm"] == 0.0 and r["coef"] == 1.0 and r["n_bad"] == 0 and len(r["norms"]) == 0


@pytest.mark.parametrize("kind", ["2", "1", "inf"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1e-44, 3e-39, 1e-30, 1e-13, 1e-10, 1e10, 1e16, 1e19, 1e30, 2e37])
def test_grad_magnitudes(peat_gpu, h, kind, dtype, scale):
    """Squares far outside float32's range, subnormal elements, a large tensor beside a tiny one."""
    import torch
    g = rng(3)
    a = (torch.randn(70001, generator=g, device="cuda", dtype=torch.float64) * scale).clamp(-3e38, 3e38).to(dt(dtype))
    b = torch.randn(300, generator=g, device="cuda").to(dt(dtype))
    mixed = b.clone()
    mixed[7] = scale
    for ts in ([a], [a, b], [b, a, mixed], [mixed]):
        want = [norm64(t, kind) for t in ts]
        r = peat_gpu.peat_grad_norm(h, ts, kind)
        for got, w in zip(r["norms"].tolist(), want):
            with np.errstate(over="ignore"):
                w32 = float(np.float32(w))  # above float32's largest the norm is infinite
            assert got == w32 if np.isinf(w32) else abs(got - w) <= TOL[kind] * w + 2.0 ** -149, (got, w)


@pytest.mark.parametrize("bad", ["propagate", "zero", "keep"])
@pytest.mark.parametrize("values", [("nan",), ("inf",), ("-inf", "nan"), ("inf", "-inf")])
def test_grad_bad_elements(peat_gpu, h, bad, values):
    import torch
    for dtype in ("f32", "f16", "bf16"):
        for kind in ("2", "1", "inf"):
            ts = grads([5000, 77, 0, 300], (dtype,), 11)
            for i, v in enumerate(values):
                ts[0][17 + 4000 * i] = float(v)
                ts[3][299 - i] = float(v)
            outs = [torch.full_like(t, 3.0) for t in ts]
            check_list(peat_gpu, h, ts, kind, 0.25, outs, 1.0, bad=bad)
            check_list(peat_gpu, h, ts, kind, 0.25, None, 1.0, bad=bad)


def test_grad_large_list_is_deterministic(peat_gpu, h):
    """More pieces than warps of a wave; the same bits on every call; in place with a factor of 1 nothing changes."""
    import torch
    sizes = [((i * 7919) % 60000) + 1 for i in range(700)] + [30_000_001]
    ts = grads(sizes, ("bf16", "f32"), 2, 1e-3)
    first = check_list(peat_gpu, h, ts)
    again = peat_gpu.peat_grad_norm(h, ts)
    assert first["norm"] == again["norm"] and np.array_equal(first["norms"], again["norms"])
    check_list(peat_gpu, h, ts, max_norm=float("inf"))
    check_list(peat_gpu, h, ts, max_norm=0.0)


def test_grad_calls_in_a_row(peat_gpu, h):
    """Long lists one after another without waiting: the staging of one call is not the next one's."""
    import torch
    lists = [grads([50 + i] * (100 + i), ("f32",), i) for i in range(9)]
    recs = [torch.zeros(16, dtype=torch.uint8, device="cuda") for _ in lists]
    for ts, r in zip(lists, recs):
        peat_gpu.peat_grad_norm_raw(h, peat_gpu.GradList(ts), r)
    for ts, r in zip(lists, recs):
        w = float(np.sqrt(sum(norm64(t, "2") ** 2 for t in ts)))
        assert abs(r.view(torch.float32)[0].item() - w) <= TOL["2"] * w


# ---------------------------------------------------------------------------
# the layer, streams, refusals
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("tnk", [(1, 40, 24), (7, 64, 48), (130, 100, 250), (600, 512, 300)])
def test_linear8(peat_gpu, h, dtype, tnk):
    """The layer's three products from the definitions, and its gradients against differences of the float64 layer:
    with g and w rounded within half a step of their scales, |dx - g w| <= sum over n of
    (|g| sw + |w| sg + sw sg / 2) / 2 (and the same for the weight), plus the result's own rounding."""
    import torch
    T, N, K = tnk
    gen = rng(T)
    x = torch.randn(T, K, generator=gen, device="cuda").to(dt(dtype))
    w = (torch.randn(N, K, generator=gen, device="cuda") / K ** 0.5).to(dt(dtype))
    g = (torch.randn(T, N, generator=gen, device="cuda")).to(dt(dtype))
    layer = peat_gpu.Linear8(h, w)
    y = layer.forward(x.view(1, T, K))
    gx, gw = layer.backward(g, x)
    assert y.shape == (1, T, N) and y.dtype == x.dtype and gx.shape == x.shape and gw.shape == w.shape

    def prod(u, v, ax):
        (qu, su, _), (qv, sv, _) = quant_definition(u, ax[0]), quant_definition(v, ax[1])
        return sums(qu, qv).float() * (su[:, None] * sv[None, :])

    assert same_bits(y[0], prod(x, w, (0, 0)).to(x.dtype))
    assert same_bits(gx, prod(g, w, (0, 1)).to(g.dtype))
    assert same_bits(gw, prod(g, x, (1, 1)))
    # L(x, w) = sum(g * (x w^T)) in binary64, by central differences along one direction each
    x64, w64, g64 = x.double(), w.double(), g.double()
    unit = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}[dtype]

    def loss(xx, ww):
        return float((g64 * (xx @ ww.t())).sum())

    e = torch.randn(T, K, generator=gen, device="cuda", dtype=torch.float64)
    f = torch.randn(N, K, generator=gen, device="cuda", dtype=torch.float64)
    step = 2.0 ** -6
    dx = (loss(x64 + step * e, w64) - loss(x64 - step * e, w64)) / (2 * step)
    dw = (loss(x64, w64 + step * f) - loss(x64, w64 - step * f)) / (2 * step)
    sg, sw = (quant_definition(v, a)[1].double() for v, a in ((g, 0), (w, 1)))
    bound = 0.5 * (g64.abs().sum(1)[:, None] * sw[None, :] + sg[:, None] * w64.abs().sum(0)[None, :]
                   + 0.5 * N * sg[:, None] * sw[None, :]) + 2 * unit * gx.double().abs()
    assert abs(float((gx.double() * e).sum()) - dx) <= float((bound * e.abs()).sum()) + 1e-6
    assert bool(((gx.double() - g64 @ w64).abs() <= bound * (1 + 1e-6) + 1e-30).all())
    sg, sx = (quant_definition(v, 1)[1].double() for v in (g, x))
    bound = 0.5 * (g64.abs().sum(0)[:, None] * sx[None, :] + sg[:, None] * x64.abs().sum(0)[None, :]
                   + 0.5 * T * sg[:, None] * sx[None, :]) + 4 * 2.0 ** -24 * gw.double().abs()
    assert abs(float((gw.double() * f).sum()) - dw) <= float((bound * f.abs()).sum()) + 1e-6
    assert bool(((gw.double() - g64.t() @ x64).abs() <= bound * (1 + 1e-6) + 1e-30).all())


def test_layer_passes_bad_values_on(peat_gpu, h):
    """A NaN in a token makes that token's outputs NaN, and every weight gradient of its channel."""
    import torch
    x = torch.randn(20, 64, generator=rng(1), device="cuda")
    w = torch.randn(48, 64, generator=rng(2), device="cuda")
    g = torch.randn(20, 48, generator=rng(3), device="cuda")
    x[3, 5] = float("nan")
    layer = peat_gpu.Linear8(h, w)
    bad = torch.isnan(layer.forward(x))
    assert bool(bad[3].all()) and int(bad.sum()) == 48
    gw = torch.isnan(layer.weight_grad(g, x))
    assert bool(gw[:, 5].all()) and int(gw.sum()) == 48


def test_other_stream(peat_gpu, h):
    """A call on a given stream is ordered there: inputs made on it, outputs read on it."""
    import torch
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        x = torch.full((64, 256), 2.0, device="cuda")
        x[:, 0] = 127.0
    q, sc = peat_gpu.peat_quantize_i8(h, x, 0, stream=s)
    y = peat_gpu.peat_matmul_i8(h, q, sc, q, sc, stream=s)
    r = peat_gpu.peat_grad_norm(h, [x], stream=s)
    s.synchronize()
    assert bool((q[:, 1:] == 2).all()) and bool((y == 127.0 ** 2 + 255 * 4).all())
    assert abs(r["norm"] - (64 * (127.0 ** 2 + 255 * 4)) ** 0.5) <= 1e-3


def test_refusals(peat_gpu, h):
    import torch
    P = peat_gpu
    x = torch.zeros(4, 8, device="cuda")
    q = torch.zeros(4, 8, dtype=torch.int8, device="cuda")
    for call in (lambda: P.peat_quantize_i8(h, x.t()), lambda: P.peat_quantize_i8(h, x.cpu()),
                 lambda: P.peat_quantize_i8(h, x[0]), lambda: P.peat_quantize_i8_raw(h, x, 0, q[:, :7]),
                 lambda: P.peat_quantize_i8_raw(h, x, 0, q, torch.zeros(3, device="cuda")),
                 lambda: P.peat_matmul_i8(h, q, None, q[:, :7], None), lambda: P.peat_matmul_i8(h, q, x[0], q, None),
                 lambda: P.peat_matmul_i8_raw(h, q, None, q, None, torch.zeros(4, 5, device="cuda")),
                 lambda: P.GradList([x], [x[:2]]), lambda: P.GradList([x], []), lambda: P.GradList([x.t()]),
                 lambda: P.GradList([x.cpu()]),
                 lambda: P.peat_grad_norm_raw(h, [x], torch.zeros(8, dtype=torch.uint8, device="cuda")),
                 lambda: P.Linear8(h, x).forward(x[:, :7])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: P.peat_quantize_i8(h, x.double()), lambda: P.peat_matmul_i8(h, x, None, x, None),
                 lambda: P.GradList([x.double()])):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(KeyError):
        P.peat_grad_norm(h, [x], norm_type="3")
    # the C boundary's own checks
    L, d = P.load(), x.data_ptr()
    rec = torch.zeros(16, dtype=torch.uint8, device="cuda").data_ptr()
    qp = q.data_ptr()

    def quant(x=d, rows=4, cols=8, ldx=8, dtype=0, axis=0, q=qp, ldq=8, scale=None, values=None, ldv=8):
        return L.peat_quantize_i8(h.ptr, x, rows, cols, ldx, dtype, axis, q, ldq, scale, values, ldv, None)

    def mm(a=qp, lda=8, sa=None, b=qp, ldb=8, sb=None, bias=None, M=4, N=4, K=8, out=d, ldo=4, t=0):
        return L.peat_matmul_i8(h.ptr, a, lda, sa, b, ldb, sb, bias, M, N, K, out, ldo, t, None)

    def clip(n=32, dtype=0, g=d, out=d, kind=0, unscale=1.0, max_norm=1.0, eps=1e-6, bad=0, result=rec, reserved=0):
        e = (P.ops.GradEntry * 1)(P.ops.GradEntry(g, out, n, dtype, reserved))
        return L.peat_grad_clip(h.ptr, e, 1, kind, unscale, max_norm, eps, bad, result, None, None)

    assert quant() == 0 and mm() == 0 and clip() == 0
    for rc in (quant(x=None), quant(rows=-1), quant(ldx=7), quant(dtype=3), quant(axis=2), quant(q=None), quant(ldq=7),
               quant(values=d, ldv=7), quant(x=d + 2), quant(scale=d + 2), mm(a=None), mm(out=None), mm(lda=7), mm(ldb=7),
               mm(ldo=3), mm(M=-1), mm(t=3), mm(t=100, sa=d), mm(out=d + 2), mm(bias=d + 1), clip(n=-1), clip(dtype=5),
               clip(g=None), clip(out=None), clip(g=d + 2), clip(kind=3), clip(unscale=0.0), clip(unscale=float("nan")),
               clip(max_norm=-1.0), clip(max_norm=float("nan")), clip(eps=-1.0), clip(eps=float("inf")), clip(bad=3),
               clip(result=None), clip(result=rec + 4), clip(reserved=1)):
        assert rc == 1
        assert P.peat_last_error(h)
    assert mm(K=131072, lda=131072, ldb=131072) == 2
    assert quant(rows=1 << 31, cols=8) == 2
    assert L.peat_grad_norm(None, None, 0, 0, 1.0, rec, None, None) == 1
    torch.cuda.synchronize()


@pytest.mark.parametrize("axes", [(0, 0), (0, 1), (1, 0), (1, 1)])
@pytest.mark.parametrize("mnk", [(1, 64, 128), (33, 70, 129), (300, 270, 520), (512, 256, 1500), (700, 300, 3100)])
@pytest.mark.parametrize("dtypes", [("f32", "bf16"), ("f16", "f16"), ("bf16", "int8"), ("int8", "f32")])
def test_product(peat_gpu, h, axes, mnk, dtypes):
    """Operands rounded on the way give what rounding and multiplying them one after the other gives."""
    import torch
    M, N, K = mnk
    g = rng(M + K)
    args, want = [], []
    for rows, axis, d in ((M, axes[0], dtypes[0]), (N, axes[1], dtypes[1])):
        if d == "int8":
            q, s = ints(rows, K, "gauss", g, 1), torch.rand(rows, generator=g, device="cuda")
            args.append((q, 0, s))
            want.append((q, s))
            continue
        x = torch.randn(rows, K, generator=g, device="cuda").to(dt(d))
        x[rows // 2] = 0.0
        x = x.t().contiguous() if axis else x
        for pad in (0, 3):
            x = torch.nn.functional.pad(x, (0, pad))[:, : x.shape[1]] if pad and rows % 2 else x
        args.append((x, axis, None))
        want.append(quant_definition(x, axis)[:2])
    (a, ax, sa), (b, bx, sb) = args
    bias = torch.randn(N, generator=g, device="cuda")
    exact = sums(want[0][0], want[1][0]).float() * (want[0][1][:, None] * want[1][1][None, :])
    for bv, out in ((None, "f32"), (bias, "bf16"), (None, "f16")):
        w = exact if bv is None else exact + bv
        got = peat_gpu.peat_product_i8(h, a, b, ax, bx, sa, sb, bv, dt(out))
        assert same_bits(got, w.to(dt(out)))


def test_product_passes_bad_values_on(peat_gpu, h):
    """NaN and infinities make their row of the operand NaN, whichever kernel takes it."""
    import torch
    for M, K in ((5, 100), (300, 200), (300, 2000)):
        x = torch.randn(M, K, generator=rng(1), device="cuda").to(torch.bfloat16)
        w = torch.randn(260, K, generator=rng(2), device="cuda").to(torch.bfloat16)
        x[M // 2, K - 1] = float("inf")
        w[77, 0] = float("nan")
        for axis in (0, 1):
            u, v = (x, w) if axis == 0 else (x.t().contiguous(), w.t().contiguous())
            y = torch.isnan(peat_gpu.peat_product_i8(h, u, v, axis, axis))
            assert bool(y[M // 2].all()) and bool(y[:, 77].all()) and int(y.sum()) == M + 260 - 1


def test_product_refusals(peat_gpu, h):
    import torch
    P, x, q = peat_gpu, torch.zeros(4, 8, device="cuda"), torch.zeros(4, 8, dtype=torch.int8, device="cuda")
    for call in (lambda: P.peat_product_i8(h, q, x, 1), lambda: P.peat_product_i8(h, x, x, a_scale=x[0, :4].contiguous()),
                 lambda: P.peat_product_i8(h, x, x[:, :7]), lambda: P.peat_product_i8(h, x, x, 0, 1),
                 lambda: P.peat_product_i8_raw(h, x, x, torch.zeros(4, 5, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        P.peat_product_i8(h, x.double(), x)
    L, O = P.load(), P.ops.Operand8

    def op(data=x.data_ptr(), rows=4, cols=8, ld=8, dtype=0, axis=0):
        return O(data, None, rows, cols, ld, dtype, axis)

    def call(a, b, t=0):
        import ctypes
        return L.peat_product_i8(h.ptr, None if a is None else ctypes.byref(a), None if b is None else ctypes.byref(b),
                                 None, x.data_ptr(), 4, t, None)
    assert call(op(), op()) == 0
    for a, b, t in ((None, op(), 0), (op(rows=-1), op(), 0), (op(ld=7), op(), 0), (op(dtype=5), op(), 0),
                    (op(axis=2), op(), 0), (op(q.data_ptr(), dtype=101, axis=1), op(), 0), (op(cols=7, ld=8), op(), 0),
                    (op(data=None), op(), 0), (op(), op(), 100), (op(), op(), 3)):
        assert call(a, b, t) == 1 and P.peat_last_error(h)
    torch.cuda.synchronize()


# ---------------------------------------------------------------------------
# sizes at which another launch shape takes over
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("axis,shape", [(0, (6001, 60)), (0, (3001, 63)), (0, (2500, 1001)), (0, (40, 1001)), (0, (3, 33001)),
                                        (1, (700, 65)), (1, (9001, 31)), (1, (513, 300)), (1, (512, 301))])
@pytest.mark.parametrize("pad", [0, 1, 5])
def test_quantize_rows_off_the_grid(peat_gpu, h, dtype, axis, shape, pad):
    """Row distances and first elements off the 16-byte grid, with few and with many rows of every length class;
    values with row distances of their own."""
    import torch
    rows, cols = shape
    g = rng(rows + cols + pad)
    off = 3 if pad else 0
    buf = torch.randn(rows * (cols + pad) + off, generator=g, device="cuda").to(dt(dtype))
    x = buf[off:].view(rows, cols + pad)[:, :cols]
    x[rows // 2, cols - 1] = float("nan")
    x[rows - 1, 0] = float("-inf")
    check_quant(peat_gpu, h, x, axis, pad, 2 * pad)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols", [1100, 2048, 2500, 4096])
def test_quantize_many_long_rows(peat_gpu, h, dtype, cols):
    """Rows enough for a warp each, longer than the shorter kernels hold."""
    import torch
    x = torch.randn(1601, cols, generator=rng(cols), device="cuda").to(dt(dtype))
    x[800, cols // 2] = float("inf")
    check_quant(peat_gpu, h, x, 0)


@pytest.mark.parametrize("axes", [(0, 0), (0, 1), (1, 0), (1, 1)])
@pytest.mark.parametrize("mnk", [(300, 513, 257), (600, 260, 2111), (1025, 300, 600)])
def test_product_off_the_grid(peat_gpu, h, axes, mnk):
    """Operands off the 16-byte grid that are rounded into the tensor cores' layout on the way."""
    import torch
    M, N, K = mnk
    g = rng(M + N + K)
    ops = []
    for rows, axis in ((M, axes[0]), (N, axes[1])):
        shape = (K, rows) if axis else (rows, K)
        buf = torch.randn(shape[0] * (shape[1] + 3) + 1, generator=g, device="cuda").to(torch.bfloat16)
        ops.append(buf[1:].view(shape[0], shape[1] + 3)[:, : shape[1]])
    want = [quant_definition(x, axis)[:2] for x, axis in zip(ops, axes)]
    exact = sums(want[0][0], want[1][0]).float() * (want[0][1][:, None] * want[1][1][None, :])
    out = torch.full((M, N + 3), 7.0, device="cuda")
    peat_gpu.peat_product_i8_raw(h, ops[0], ops[1], out[:, :N], *axes)
    assert same_bits(out[:, :N], exact) and bool((out[:, N:] == 7).all())


def test_quantize_and_product_sizes_in_turn(peat_gpu, h):
    """Column maxima and sums of squares live in two halves of a workspace, used and cleared in turn by calls of
    different sizes: a large matrix leaves nothing behind for a small one."""
    import torch
    g = rng(77)
    xs = [(torch.randn(r, c, generator=g, device="cuda") * s).to(torch.bfloat16)
          for r, c, s in ((600, 900, 1e4), (2000, 40, 1e-3), (700, 20000, 1e3), (515, 9, 1.0), (600, 900, 1e-2))]
    pairs = [(torch.randn(M, K, generator=g, device="cuda") * s, torch.randn(N, K, generator=g, device="cuda"))
             for M, N, K, s in ((600, 300, 5000, 1.0), (300, 260, 1500, 1e-3), (900, 500, 9000, 1.0))]
    for _ in range(3):
        got = []
        for i, x in enumerate(xs):
            got.append(peat_gpu.peat_quantize_i8(h, x, 1))
            a, b = pairs[i % 3]
            got.append(peat_gpu.peat_product_i8(h, a, b))
        for i, x in enumerate(xs):
            q, s, _ = quant_definition(x, 1)
            assert torch.equal(got[2 * i][0], q) and same_bits(got[2 * i][1], s)
            a, b = (quant_definition(t, 0)[:2] for t in pairs[i % 3])
            assert same_bits(got[2 * i + 1], sums(a[0], b[0]).float() * (a[1][:, None] * b[1][None, :]))


# ---------------------------------------------------------------------------
# lists longer than a kernel argument holds, waits that expire
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("count", [96, 97, 800, 801, 2500])
def test_grad_long_lists(peat_gpu, h, count):
    """As many tensors as travel with the launch, one more, and many more, clipped in place and elsewhere."""
    import torch
    ts = grads([(i * 37) % 301 for i in range(count)], ("bf16", "f32", "f16"), count, 0.1)
    check_list(peat_gpu, h, ts, max_norm=0.5, outs=[torch.empty_like(t) for t in ts])
    check_list(peat_gpu, h, ts, max_norm=0.5)


def test_grad_long_lists_in_a_row(peat_gpu, h):
    """More calls than staging buffers, the lists growing and shrinking, with nothing waiting between them."""
    import torch
    lists = [grads([20 + i] * (801 + 300 * (i % 5)), ("f32",), i) for i in range(11)]
    recs = [torch.zeros(16, dtype=torch.uint8, device="cuda") for _ in lists]
    glists = [peat_gpu.GradList(ts) for ts in lists]
    torch.cuda._sleep(20_000_000)
    for ts, r in zip(glists, recs):
        peat_gpu.peat_grad_norm_raw(h, ts, r)
    for ts, r in zip(lists, recs):
        w = norm64(torch.cat(ts), "2")
        assert abs(r.view(torch.float32)[0].item() - w) <= TOL["2"] * w


def test_expired_wait_is_reported(peat_gpu, h):
    """A handle whose bounded waits give up at once: the product returns, the next one reports it, and other handles
    go on."""
    import torch
    g = rng(3)
    a, b = ints(2100, 1024, "uniform", g), ints(2060, 1024, "uniform", g)
    out = torch.empty(2100, 2060, dtype=torch.int32, device="cuda")
    bad = peat_gpu.Handle(0, flags=peat_gpu.PEAT_FLAG_TEST_EXPIRE_WAITS)
    for _ in range(2):
        peat_gpu.peat_matmul_i8_raw(bad, a, None, b, None, out)
        torch.cuda.synchronize()
        with pytest.raises(peat_gpu.PeatError) as e:
            peat_gpu.peat_matmul_i8_raw(bad, a, None, b, None, out)
        assert e.value.status == 5
    bad.close()
    peat_gpu.peat_matmul_i8_raw(h, a, None, b, None, out)
    assert torch.equal(out.to(torch.int64), sums(a, b))


@pytest.mark.parametrize("mnk", [(1, 8192, 64), (5, 8200, 700), (9, 9001, 131), (16, 20000, 260), (17, 8193, 1025), (33, 8192, 1500),
                                 (64, 8210, 4200)])
def test_matmul_few_rows_past_many(peat_gpu, h, mnk):
    """Few rows of a past many of b, the runs of a tile shared by several warps, with rows on the 16-byte grid and off it."""
    import torch
    M, N, K = mnk
    g = rng(sum(mnk))
    for pad in (-K % 16, 3 - K % 2):
        a, b = ints(M, K, "uniform", g, pad), ints(N, K, "uniform", g, pad)
        out = torch.empty(M, N, dtype=torch.int32, device="cuda")
        peat_gpu.peat_matmul_i8_raw(h, a, None, b, None, out)
        assert torch.equal(out.to(torch.int64), sums(a, b))


# ---------------------------------------------------------------------------
# graphs
# ---------------------------------------------------------------------------
def test_captured_calls(peat_gpu):
    """Calls captured into a graph and replayed on new inputs, between calls that are not, and after the workspace has
    grown."""
    import torch
    P, g = peat_gpu, rng(21)
    with P.Handle(0) as h:
        x = torch.empty(900, 700, device="cuda", dtype=torch.bfloat16)
        a, b = torch.empty(600, 2100, device="cuda"), torch.empty(300, 2100, device="cuda")
        at, bt = torch.empty(1300, 270, device="cuda"), torch.empty(1300, 280, device="cuda")
        grads_in = [torch.empty(n, device="cuda") for n in (5, 70000, 1000)]
        grads_out = [torch.empty_like(t) for t in grads_in]
        q, s = torch.empty(700, 900, dtype=torch.int8, device="cuda"), torch.empty(700, device="cuda")
        y, yt = torch.empty(600, 300, device="cuda"), torch.empty(270, 280, device="cuda")
        rec, norms = torch.empty(16, dtype=torch.uint8, device="cuda"), torch.empty(3, device="cuda")
        glist = P.GradList(grads_in, grads_out)

        def refill(scale):
            for t in (x, a, b, at, bt, *grads_in):
                t.copy_(torch.randn(t.shape, generator=g, device="cuda") * scale)

        def calls():
            P.peat_quantize_i8_raw(h, x, 1, q, s)
            P.peat_product_i8_raw(h, a, b, y)
            P.peat_product_i8_raw(h, at, bt, yt, 1, 1)
            P.peat_grad_clip_raw(h, glist, 0.5, rec, norms)

        def check():
            torch.cuda.synchronize()
            eq, es, _ = quant_definition(x, 1)
            assert torch.equal(q, eq) and same_bits(s, es)
            for u, v, w, axis in ((a, b, y, 0), (at, bt, yt, 1)):
                (qu, su, _), (qv, sv, _) = quant_definition(u, axis), quant_definition(v, axis)
                assert same_bits(w, sums(qu, qv).float() * (su[:, None] * sv[None, :]))
            r = rec.view(torch.float32)
            want = norm64(torch.cat(grads_in), "2")
            assert abs(r[0].item() - want) <= TOL["2"] * want
            for t, o in zip(grads_in, grads_out):
                assert same_bits(o, t * r[1])

        refill(1.0)
        calls()
        check()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls()
        for scale in (100.0, 1e-3, 5.0):
            refill(scale)
            graph.replay()
            check()
            refill(scale * 3)
            calls()
            check()
        big = torch.randn(1100, 40000, generator=g, device="cuda")  # larger than any call before
        P.peat_quantize_i8(h, big, 1)
        P.peat_product_i8(h, big, big[:300])
        P.peat_grad_norm(h, [torch.ones(10, device="cuda")] * 5000)
        for scale in (7.0, 1e-2):
            refill(scale)
            graph.replay()
            check()


def test_capture_refusals(peat_gpu):
    """A capture that would have to allocate is refused, and the handle works on."""
    import torch
    P = peat_gpu
    x = torch.randn(700, 64, generator=rng(4), device="cuda")
    q, s = torch.empty(64, 700, dtype=torch.int8, device="cuda"), torch.empty(64, device="cuda")
    rec = torch.empty(16, dtype=torch.uint8, device="cuda")
    long = P.GradList([torch.ones(3, device="cuda") for _ in range(801)])
    with P.Handle(0) as h:
        for warm in (False, True):
            if warm:
                P.peat_quantize_i8_raw(h, x, 1, q, s)
                P.peat_grad_norm_raw(h, long, rec)
                torch.cuda.synchronize()
            done = torch.zeros(1, device="cuda")
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                done.add_(1)
                if not warm:
                    with pytest.raises(P.PeatError) as e:
                        P.peat_quantize_i8_raw(h, x, 1, q, s)
                    assert e.value.status == 2
                with pytest.raises(P.PeatError) as e:
                    P.peat_grad_norm_raw(h, long, rec)
                assert e.value.status == 2
            graph.replay()
            torch.cuda.synchronize()
            assert done.item() == 1
        check_quant(P, h, x, 1)
        assert abs(P.peat_grad_norm(h, long)["norm"] - 2403 ** 0.5) <= 1e-4


@pytest.mark.parametrize("mnk", [(777, 1000, 2049), (600, 520, 20000)])
def test_expired_wait_in_split_tiles(peat_gpu, h, mnk):
    """The same where two or four CTA pairs of a cluster share a tile: all of them meet and end."""
    import torch
    M, N, K = mnk
    g = rng(4)
    a, b = ints(M, K, "uniform", g, -K % 16), ints(N, K, "uniform", g, -K % 16)
    out = torch.empty(M, N, dtype=torch.int32, device="cuda")
    bad = peat_gpu.Handle(0, flags=peat_gpu.PEAT_FLAG_TEST_EXPIRE_WAITS)
    for _ in range(2):
        peat_gpu.peat_matmul_i8_raw(bad, a, None, b, None, out)
        torch.cuda.synchronize()
        with pytest.raises(peat_gpu.PeatError) as e:
            peat_gpu.peat_matmul_i8_raw(bad, a, None, b, None, out)
        assert e.value.status == 5
    bad.close()
    peat_gpu.peat_matmul_i8_raw(h, a, None, b, None, out)
    assert torch.equal(out.to(torch.int64), sums(a, b))


@pytest.mark.parametrize("K", [1, 15, 63, 1001, 4099])
def test_one_row_against_many(peat_gpu, h, K):
    """One row, whose distance to the next is nothing to go by, against padded rows, on either side; its integers from a
    buffer of exactly their length."""
    import torch
    g = rng(K)
    x = torch.randn(1, K, generator=g, device="cuda")
    guard = torch.full((K + 16,), 55, dtype=torch.int8, device="cuda")
    q, scale = guard[:K].view(1, K), torch.empty(1, device="cuda")
    peat_gpu.peat_quantize_i8_raw(h, x, 0, q, scale)
    eq, es, _ = quant_definition(x, 0)
    assert torch.equal(q, eq) and same_bits(scale, es) and bool((guard[K:] == 55).all())
    peat_gpu.peat_quantize_i8_raw(h, x.view(K, 1), 1, q, scale)
    assert torch.equal(q, eq) and same_bits(scale, es) and bool((guard[K:] == 55).all())
    for rows in (1, 7, 600, 9000):
        b = ints(rows, K, "uniform", g, -K % 16)
        for u, v in ((q, b), (b, q)):
            buf = torch.full((u.shape[0] + 1, v.shape[0] + 3), -5, dtype=torch.int32, device="cuda")
            out = buf[: u.shape[0], : v.shape[0]]
            peat_gpu.peat_matmul_i8_raw(h, u, None, v, None, out)
            assert torch.equal(out.to(torch.int64), sums(u, v))
            assert bool((buf[u.shape[0]:] == -5).all()) and bool((buf[:, v.shape[0]:] == -5).all())


def test_layer_takes_any_strides(peat_gpu, h):
    """Transposed, sliced and expanded tensors (a broadcast sum's gradient among them) give what their copies give, two
    dimensions like three."""
    import torch
    g = rng(31)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)
    xs = [normal(64, 40).t(), normal(5, 8, 128)[:, :, ::2], normal(40, 1).expand(40, 64), normal(64).expand(5, 8, 64),
          normal(8, 5, 64).transpose(0, 1), normal(1, 1).expand(40, 64)]
    gs = [normal(48, 40).t(), normal(5, 8, 96)[:, :, 48:], normal(48).expand(40, 48), normal(1, 1, 1).expand(5, 8, 48),
          normal(8, 5, 48).transpose(0, 1), normal(48, 40).t()]
    w = normal(64, 48).t()
    layer, want = peat_gpu.Linear8(h, w), peat_gpu.Linear8(h, w.contiguous())
    for x, dy in zip(xs, gs):
        xc, dc = x.contiguous(), dy.contiguous()
        assert same_bits(layer.forward(x), want.forward(xc))
        for got, expected in zip(layer.backward(dy, x), want.backward(dc, xc)):
            assert same_bits(got, expected)


def test_layer_without_inputs(peat_gpu, h):
    """No features in, or no tokens."""
    import torch
    layer = peat_gpu.Linear8(h, torch.zeros(48, 0, device="cuda"))
    x, dy = torch.zeros(2, 3, 0, device="cuda"), torch.ones(2, 3, 48, device="cuda")
    y, (dx, dw) = layer.forward(x), layer.backward(dy, x)
    assert y.shape == (2, 3, 48) and not y.any() and dx.shape == (2, 3, 0) and dw.shape == (48, 0)
    layer = peat_gpu.Linear8(h, torch.ones(48, 64, device="cuda"))
    for shape in ((0,), (2, 0)):
        x, dy = torch.zeros(*shape, 64, device="cuda"), torch.ones(*shape, 48, device="cuda")
        y, (dx, dw) = layer.forward(x), layer.backward(dy, x)
        assert y.shape == (*shape, 48) and dx.shape == (*shape, 64) and dw.shape == (48, 64) and not dw.any()


def test_grad_outputs_of_the_same_order(peat_gpu, h):
    """An output lies in memory as its gradient does, whatever the strides of dimensions of size 1 say; another order is
    refused."""
    import torch
    g = rng(8)
    last = torch.channels_last
    one = torch.randn(6, 5, 1, 1, generator=g, device="cuda").as_strided((6, 5, 1, 1), (5, 1, 5, 5))
    full = torch.randn(6, 5, 3, 2, generator=g, device="cuda").to(memory_format=last)
    deep = torch.randn(6, 1, 3, 2, generator=g, device="cuda").to(memory_format=last)
    ts = [one, full, deep]
    outs = [torch.empty(6, 5, 1, 1, device="cuda"), torch.empty_like(full), torch.empty(6, 1, 3, 2, device="cuda")]
    r = peat_gpu.peat_grad_clip(h, peat_gpu.GradList(ts, outs), 0.5)
    for t, o in zip(ts, outs):
        assert torch.equal(o, t * np.float32(r["coef"]))
    for t, o in ((full, torch.empty(6, 5, 3, 2, device="cuda")), (full.contiguous(), torch.empty_like(full))):
        with pytest.raises(ValueError):
            peat_gpu.GradList([t], [o])


@pytest.mark.parametrize("fill", ["low", "high", "gauss", "uniform"])
@pytest.mark.parametrize("mnk", [(2500, 2500, 2000), (5000, 4700, 2100), (4800, 1000, 9000)])
def test_matmul_long_sums_of_many_tiles(peat_gpu, h, fill, mnk):
    """Sums that leave the accumulator in several pieces where no tile is split: one or two tiles a CTA pair, five of them
    (more than are planned ahead), and pieces past the first 32 norm blocks."""
    import torch
    M, N, K = mnk
    g = rng(M + K)
    a, b = ints(M, K, fill, g, -K % 16), ints(N, K, fill, g, -K % 16)
    if fill == "gauss":  # some rows and some stretches of k that need their pieces, others that do not
        a[: M // 2].fill_(-128)
        b[:, : K // 2].fill_(127)
    want = sums(a, b)
    sa, sb = torch.rand(M, generator=g, device="cuda"), torch.rand(N, generator=g, device="cuda")
    scaled = want.float() * (sa[:, None] * sb[None, :])
    out = torch.empty(M, N, dtype=torch.int32, device="cuda")
    for _ in range(2):
        out.fill_(-1)
        peat_gpu.peat_matmul_i8_raw(h, a, None, b, None, out)
        assert torch.equal(out, want.int())
    assert same_bits(peat_gpu.peat_matmul_i8(h, a, sa, b, sb), scaled)
