"""The 4-bit products, the 8-bit layer behind the norm, and the norm's gradients: strides, row counts, lengths and empty
matrices at the edges of what the calls allow, against the definitions in 64 bits."""
import pytest
import test_gpu_ops4 as T

pytestmark = pytest.mark.gpu

EPS = T.EPS


@pytest.fixture(scope="module")
def h(peat_gpu):
    handle = peat_gpu.Handle(0)
    yield handle
    handle.close()


@pytest.mark.parametrize("lead,width,features,out", [((100, 3000), 32, 4, "bf16"), ((5, 26), 200, 1, "f32"), ((65, 2), 96, 40, "bf16"),
                                                     ((60, 100), 64, 40, "f32")])
def test_rounded_input_of_turned_dimensions(peat_gpu, h, lead, width, features, out):
    """q and scale with their leading dimensions in another order than memory's give what contiguous ones give: the copy of
    the scales outlives the call, also where the results would fit its place (300 000 rows, in several waves)."""
    import torch
    g = T.rng(width)
    layer = peat_gpu.Linear8(h, torch.randn(features, width, generator=g, device="cuda"))
    q = torch.randint(-127, 128, (*lead, width), generator=g, device="cuda", dtype=torch.int8)
    scale = torch.rand(*lead, generator=g, device="cuda")
    flat_q, flat_scale = q.transpose(0, 1).contiguous(), scale.transpose(0, 1).contiguous()
    want = layer.forward_rounded(flat_q, flat_scale, T.dt(out))
    for _ in range(3):
        torch.cuda.empty_cache()  # (what a call frees is then the first place that its next tensor finds)
        y = layer.forward_rounded(q.transpose(0, 1), scale.transpose(0, 1), T.dt(out))
        assert y.shape == (lead[1], lead[0], features) and T.same_bits(y, want)


@pytest.mark.parametrize("dtype", T.DTYPES)
@pytest.mark.parametrize("format", T.FORMATS)
@pytest.mark.parametrize("rows", [1, 15, 77, 129, 4097])
@pytest.mark.parametrize("cols", [64, 128])
def test_quantize_rows_of_half_a_warp(peat_gpu, h, dtype, format, rows, cols):
    """Rows of 16 vectors, two to a warp, and an odd number of them: the last warp has a row of the matrix and one that is
    not."""
    import torch
    for pad in (0, 8):
        x = torch.randn(rows, cols + pad, generator=T.rng(rows), device="cuda").to(T.dt(dtype))[:, :cols]
        T.check_quant(peat_gpu, h, x, format, 0, 0, pad)


def test_rmsnorm_backward_of_the_widest_rows(peat_gpu, h):
    """2^27 columns, the most that the call takes, in the type that has the most pieces a row."""
    import torch
    cols, g = 1 << 27, T.rng(27)
    x, grad = torch.randn(1, cols, generator=g, device="cuda"), torch.rand(1, cols, generator=g, device="cuda")
    w, rstd = torch.rand(cols, generator=g, device="cuda") + 0.5, torch.full((1,), 1.25, device="cuda")
    dx, dw = peat_gpu.peat_rmsnorm_backward(h, grad, x, w, rstd)
    n, d = x.double() * 1.25, grad.double()
    assert bool(((dw.double() - (d * n)[0]).abs() <= 2 * EPS * (d * n)[0].abs()).all())
    gn = d * w.double() * n
    c, size = gn.mean(), gn.abs().mean()
    del gn
    # a product's 3 roundings and 4 more in its vector, 64 vectors; 2^17 vectors a thread one after the other, those
    # additions' errors kept, to the square of as many roundings; 13 partial sums and the division
    off = ((3 + 4 + 64 + 14) * EPS + (2.0 ** 17 * EPS) ** 2) * size
    want = 1.25 * (d * w.double() - n * c)
    tol = 1.25 * (n.abs() * off + 5 * EPS * ((d * w.double()).abs() + (n * c).abs())) + EPS * want.abs()
    assert bool(((dx.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("more,pad,off", [(3, 5, 0), (3, 5, 1), (8, 8, 0)])
def test_rmsnorm_backward_sums_of_long_rows(peat_gpu, h, dtype, more, pad, off):
    """A row's inner product over 2^24 elements of one sign, whose single additions all round the same way: grad_x is what
    is left of g and of that mean, which cancel."""
    import torch
    cols = (1 << 24) + more
    t, w = T.dt(dtype), torch.full((cols,), 0.7, device="cuda")
    rstd = torch.ones(2, device="cuda")
    buf = torch.ones(2 * (cols + pad) + off, device="cuda", dtype=t)
    x = buf[off:].view(2, cols + pad)[:, :cols]
    grad = torch.empty(2, cols, device="cuda", dtype=t)
    grad[0], grad[1] = 0.1, 0.7
    dx, dw = peat_gpu.peat_rmsnorm_backward(h, grad, x, w, rstd)
    assert torch.equal(dw, grad.float()[0] + grad.float()[1])
    # (g is constant and n = 1: c is that constant)  8 products of 2 roundings and an addition each in a vector; 2^13
    # (float32 2^14) vectors a thread one after the other with their errors kept, to the square of as many roundings, or
    # (float32 on the grid) 64 of them before that; 13 partial sums and the division; then g's own rounding, the
    # difference, the product by rstd
    g = 0.7 * grad[:, :1].double()
    vectors = 2.0 ** (13 if dtype == "bf16" else 14) + 1
    run = 64 if (dtype, more) == ("f32", 8) else 0
    tol = ((8 + 2 + 2 + run + 14) * EPS + (vectors * EPS) ** 2) * g + 5 * EPS * g
    assert float((dx.double().abs() - tol).max()) <= 0.0


@pytest.mark.parametrize("m", [3, 300])
def test_4_bit_products_of_no_k_look_at_no_scale(peat_gpu, h, m):
    """Without k the results are 0, plus the bias, whatever the rows' scales hold."""
    import torch
    bad = torch.tensor([float("nan"), float("inf"), 1.0], device="cuda")
    empty = lambda rows, scale: peat_gpu.Float4("nvfp4", torch.empty(rows, 0, dtype=torch.uint8, device="cuda"),
                                                torch.empty(0, dtype=torch.uint8, device="cuda"), scale)
    a, b = empty(m, bad.repeat(m // 3)), empty(300, bad.repeat(100))
    bias = torch.randn(300, generator=T.rng(m), device="cuda")
    for bv, want in ((bias, bias.expand(m, 300)), (None, torch.zeros(m, 300, device="cuda"))):
        assert torch.equal(peat_gpu.peat_matmul_f4(h, a, b, bv), want)
        assert torch.equal(peat_gpu.peat_product_f4(h, a, b, None, 0, 0, bv), want)


@pytest.mark.parametrize("m", [3, 300])
def test_8_bit_products_of_no_k_look_at_no_scale(peat_gpu, h, m):
    import torch
    bad = torch.tensor([float("nan"), float("inf"), 1.0], device="cuda")
    sa, sb = bad.repeat(m // 3), bad.repeat(100)
    a, b = (torch.empty(rows, 0, dtype=torch.int8, device="cuda") for rows in (m, 300))
    bias = torch.randn(300, generator=T.rng(m), device="cuda")
    for bv, want in ((bias, bias.expand(m, 300)), (None, torch.zeros(m, 300, device="cuda"))):
        assert torch.equal(peat_gpu.peat_matmul_i8(h, a, sa, b, sb, bv), want)
        assert torch.equal(peat_gpu.peat_product_i8(h, a, b, 0, 0, sa, sb, bv), want)


def test_norm_of_no_columns(peat_gpu, h):
    """Rows of nothing: a mean of nothing is no number, a largest of nothing 0; the layer behind them gives its bias."""
    import torch
    x, w = torch.empty(5, 3, 0, device="cuda"), torch.empty(0, device="cuda")
    scale, rstd = torch.full((15,), 7.0, device="cuda"), torch.full((15,), 7.0, device="cuda")
    peat_gpu.peat_rmsnorm_raw(h, x.view(15, 0), w, scale=scale, rstd=rstd)
    assert not bool(scale.any()) and bool(torch.isnan(rstd).all())
    got = peat_gpu.RMSNorm8(h, w).forward(x)
    assert got["q"].shape == x.shape and not bool(got["scale"].any()) and bool(torch.isnan(got["rstd"]).all())
    bias = torch.randn(40, generator=T.rng(1), device="cuda")
    y = peat_gpu.Linear8(h, torch.empty(40, 0, device="cuda")).forward_rounded(got["q"], got["scale"], bias=bias)
    assert torch.equal(y, bias.expand(5, 3, 40))


@pytest.mark.parametrize("format", T.FORMATS)
def test_values_of_an_empty_matrix(peat_gpu, h, format):
    import torch
    for rows, cols in ((0, 64), (0, 0), (5, 0), (130, 0)):
        f = peat_gpu.peat_quantize_f4(h, torch.empty(rows, cols, device="cuda"), format)
        assert f.values().shape == (rows, cols) and f.values().dtype == torch.float32


@pytest.mark.parametrize("dtype", T.DTYPES)
@pytest.mark.parametrize("cols", [40, 1001, 4096, 20000])
def test_rmsnorm_backward_rounds_as_documented(peat_gpu, h, dtype, cols):
    """rstd (g - n c) + grad_sum: the first difference is one fused operation, the others are rounded one by one.  Where
    x = 0 (c = 0) that leaves grad weight, its product by rstd and the sum, bit for bit."""
    import torch
    g = T.rng(cols)
    grad, add = (torch.randn(64, cols, generator=g, device="cuda").to(T.dt(dtype)) for _ in range(2))
    w, rstd = (torch.rand(n, generator=g, device="cuda") + 0.5 for n in (cols, 64))
    dx, dw = peat_gpu.peat_rmsnorm_backward(h, grad, torch.zeros_like(grad), w, rstd, add)
    want = T.single(T.single(grad.double() * w.double()) * rstd.double()[:, None])
    assert T.same_values(dx, (want + add.double()).float().to(dx.dtype)) and not bool(dw.any())
    alone = peat_gpu.peat_rmsnorm_backward(h, grad, torch.zeros_like(grad), w, rstd)[0]
    assert T.same_values(alone, want.to(dx.dtype))
