"""Layer norm's rows in full: statistics of rows with Inf and NaN, batches of many rows, rows wherever they lie."""
import pytest
import torch

from paper_2112_10769_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [5, 64, 300, 1000, 1024, 4096, 9001, 40000])
def test_the_statistics_of_rows_with_inf_and_nan_are_the_formulas(ctx, cols, dtype):
    # mean: Inf with its sign, NaN for NaN or for both infinities; rstd: NaN, for the variance is
    x = torch.randn(7, cols, device="cuda").to(dtype)
    clean = ctx.layer_norm(x)
    x[1, 2], x[3, cols - 1], x[4, 0], x[5, 1], x[5, cols - 1] = float("inf"), float("nan"), -float("inf"), float("inf"), -float("inf")
    y, mean, rstd = ctx.layer_norm(x)
    for got, before in zip((y, mean, rstd), clean):
        assert torch.equal(got[[0, 2, 6]], before[[0, 2, 6]])
    bad = [1, 3, 4, 5]
    assert torch.isnan(y[bad]).all() and torch.isnan(rstd[bad]).all()
    assert mean[1] == float("inf") and mean[4] == -float("inf") and torch.isnan(mean[[3, 5]]).all()


# ---- training batches and prompts: many rows a group ------------------------------------------------------------
# Tolerances, u = 2^-24.  A row's sums are at most cols / 32 additions in a thread and a tree (c = 32 + cols / 32
# roundings, relative to the largest terms); bf16 results add one rounding, 2^-8 of the value with a factor of two to
# spare.  A column's sum is at most rows / SMs additions in a group, then at most 32 groups or warps of a block and at most
# 32 + 5 additions over the blocks, of terms with at most 10 roundings: d = 80 + rows / SMs roundings.  One row left out
# or taken twice moves a column's sum by about 1 / rows of the sum of magnitudes, which is more than that for every
# shape here (1.1 times for 41582 rows, 4 for 20000, 38 for 4099).
U, EPS = 2.0 ** -24, 1e-5
BATCHES = [(4099, 771, 5, 0), (4099, 771, 0, 1), (20000, 301, 0, 0), (20000, 320, 0, 0), (30000, 128, 0, 0), (9001, 187, 3, 1),
           (41582, 704, 0, 0), (12000, 768, 0, 0), (12001, 700, 0, 0), (6000, 1024, 0, 0), (5000, 1025, 0, 1), (9000, 1536, 8, 0),
           (6000, 4096, 0, 0), (5223, 3830, 0, 0), (3000, 6144, 0, 0), (2500, 9001, 0, 0), (2400, 12288, 0, 0), (1300, 16384, 0, 0),
           (1201, 20000, 0, 0), (1201, 20001, 3, 1)]


def batch(rows, cols, pad, shift, dtype, seed):
    """[rows, cols] with a row stride of cols + pad, `shift` elements into its storage; every row another size and mean."""
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn(rows * (cols + pad) + shift, device="cuda", generator=g)[shift:].view(rows, cols + pad)
    x *= torch.exp(torch.randn(rows, 1, device="cuda", generator=g))
    x += torch.randn(rows, 1, device="cuda", generator=g)
    if dtype == torch.float32:
        return x[:, :cols]
    flat = torch.empty(rows * (cols + pad) + shift, device="cuda", dtype=dtype)
    flat[shift:].view(rows, cols + pad).copy_(x)
    return flat[shift:].view(rows, cols + pad)[:, :cols]


def parameters(cols):
    g = torch.Generator("cuda").manual_seed(cols)
    return 1 + 0.3 * torch.randn(cols, device="cuda", generator=g), 0.2 * torch.randn(cols, device="cuda", generator=g)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,pad,shift", BATCHES)
def test_batches_against_64_bits(ctx, rows, cols, pad, shift, dtype):
    x = batch(rows, cols, pad, shift, dtype, 1)
    w, b = parameters(cols)
    c = 32 + cols / 32
    rounded = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    x64 = x.double()
    m64 = x64.mean(1, keepdim=True)
    d = x64 - m64
    r64 = (d.square().mean(1, keepdim=True) + EPS).rsqrt()
    spread = d.abs().amax(1, keepdim=True)
    y, mean, rstd = ctx.layer_norm(x, w, b, EPS)
    assert ((mean.double() - m64[:, 0]).abs() <= c * U * (m64.abs() + spread)[:, 0]).all()
    assert ((rstd.double() - r64[:, 0]).abs() <= c * U * r64[:, 0]).all()
    y64 = d * r64 * w.double() + b.double()
    size = spread * r64 * w.double().abs() + b.double().abs()
    assert ((y.double() - y64).abs() <= c * U * size + rounded * y64.abs()).all()
    # the norm's result as codes: half a step, what the value is off, and the factor's and product's roundings
    q, s = ctx.layer_norm_int8(x, w, b, EPS)
    err = c * U * size
    s64 = y64.abs().amax(1) / 127
    assert ((s.double() - s64).abs() <= err.amax(1) / 127 + 2 * U * s64).all()
    assert ((q.double() * s.double()[:, None] - y64).abs() <= (0.5 + 4 * 127 * U) * s.double()[:, None] + 2 * err).all()
    del y, y64, size, err, d, q
    # the codes of the rows themselves: the definition, binary32 operation by operation
    q, s = ctx.quant_int8_rows(x)
    top = x.float().abs().amax(1)
    factor = torch.full_like(top, 127) * (torch.ones_like(top) / top)
    assert torch.equal(s, top / torch.full_like(top, 127))
    assert torch.equal(q, (x.float() * factor[:, None]).round().to(torch.int8))
    del q
    # backward, with the mean and 1/std that it is given
    dy = batch(rows, cols, pad, shift, dtype, 2)
    dx, dw, db = ctx.layer_norm_bwd(dy, x, mean, rstd, w)
    r, xhat, dy64 = rstd.double()[:, None], (x64 - mean.double()[:, None]) * rstd.double()[:, None], dy.double()
    g = dy64 * w.double()
    along = (g * xhat).mean(1, keepdim=True)
    dx64 = r * (g - g.mean(1, keepdim=True) - xhat * along)
    size = r * (g.abs() + g.abs().mean(1, keepdim=True) + xhat.abs() * (g * xhat).abs().mean(1, keepdim=True))
    assert ((dx.double() - dx64).abs() <= c * U * size + rounded * dx64.abs()).all()
    n = 80 + rows / torch.cuda.get_device_properties(0).multi_processor_count
    assert ((dw.double() - (dy64 * xhat).sum(0)).abs() <= n * U * (dy64 * xhat).abs().sum(0)).all()
    assert ((db.double() - dy64.sum(0)).abs() <= n * U * dy64.abs().sum(0)).all()
    only = ctx.layer_norm_bwd(dy, x, mean, rstd, w, need_dx=False)
    assert only[0] is None and torch.equal(only[1], dw) and torch.equal(only[2], db)
    assert ctx.status() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(3000, 96), (3000, 301), (3000, 512), (3000, 704), (3000, 771), (2000, 1024), (2000, 3830), (2000, 4096),
                                       (1500, 9001), (1300, 16384), (700, 20000)])
def test_a_row_does_not_depend_on_the_others_nor_on_where_it_lies(ctx, rows, cols, dtype):
    x, dy = (batch(rows, cols, 0, 0, dtype, i) for i in (1, 2))
    w, b = parameters(cols)

    def results(x, dy):
        y, mean, rstd = ctx.layer_norm(x, w, b, EPS)
        return (y, mean, rstd, *ctx.layer_norm_int8(x, w, b, EPS), *ctx.quant_int8_rows(x),
                ctx.layer_norm_bwd(dy, x, mean, rstd, w, need_dweight=False, need_dbias=False)[0])

    want = results(x, dy)

    def moved(t, pad, shift):
        flat = torch.empty(t.shape[0] * (cols + pad) + shift, device="cuda", dtype=dtype)
        view = flat[shift:].view(t.shape[0], cols + pad)[:, :cols]
        return view.copy_(t)

    for first, last in ((0, 1), (rows - 1, rows), (rows // 2, rows // 2 + 7), (1, 400), (0, rows)):
        for pad, shift in ((0, 0), (8, 0), (3, 1)):
            for a, whole in zip(results(moved(x[first:last], pad, shift), moved(dy[first:last], pad, shift)), want):
                assert torch.equal(a, whole[first:last])
    assert ctx.status() == 0
