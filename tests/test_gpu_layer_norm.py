"""Layer norm, forward and backward, and the row-wise int8 quantizer, against plain forms in 64 bits.

Tolerances.  u = 2^-24.  A row's sums are made of at most cols / 32 sequential additions per thread and a tree,
so a mean of values of size A is off by at most c u A with c = 32 + cols / 32; bf16 results add one
rounding, 2^-8 of the value (generous by a factor of two)."""
import numpy as np
import pytest
import torch

from paper_2112_10769_b200 import binding

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-5


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def make(rows, cols, dtype, seed, pad=0, shift=0, mean=0.5):
    """[rows, cols] with a row stride of cols + pad, starting `shift` elements into its storage."""
    g = torch.Generator("cuda").manual_seed(seed)
    flat = torch.randn(rows * (cols + pad) + shift, device="cuda", generator=g) * 2 + mean
    return flat.to(dtype)[shift:].view(rows, cols + pad)[:, :cols]


def norm64(x, w, b, eps=EPS):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = (d.square().mean(1, keepdim=True) + eps).rsqrt()
    y = d * rstd
    if w is not None:
        y = y * w.double()
    if b is not None:
        y = y + b.double()
    size = d.abs().amax(1, keepdim=True) * rstd * (1 if w is None else w.double().abs()) + (0 if b is None else b.double().abs())
    return y, mean[:, 0], rstd[:, 0], size, d.abs().amax(1)


def params(cols, seed, which):
    g = torch.Generator("cuda").manual_seed(seed)
    w = 1 + 0.3 * torch.randn(cols, device="cuda", generator=g)
    b = 0.2 * torch.randn(cols, device="cuda", generator=g)
    return (w if which & 1 else None), (b if which & 2 else None)


SHAPES = [(1, 1), (1, 2), (3, 7), (1, 1024), (5, 31), (4, 32), (2, 33), (7, 255), (9, 256), (3, 257), (6, 512), (17, 771),
          (64, 1000), (33, 1024), (5, 1025), (3, 2047), (4, 2048), (300, 96), (2, 4095), (3, 4096), (2, 5000), (2, 8192),
          (1, 12288), (2, 16384), (2, 16385), (2, 33000), (1, 70001), (1000, 64), (2500, 16), (700, 5)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_forward(ctx, rows, cols, dtype):
    for pad, shift, which in ((0, 0, 3), (5, 0, 1), (8, 0, 3), (0, 1, 2), (3, 3, 0)):
        x = make(rows, cols, dtype, rows * 31 + cols + pad, pad, shift)
        w, b = params(cols, cols, which)
        y, mean, rstd = ctx.layer_norm(x, w, b, EPS)
        y64, m64, r64, size, spread = norm64(x, w, b)
        c = 32 + cols / 32
        assert y.dtype == dtype and y.shape == x.shape
        assert ((mean.double() - m64).abs() <= c * U * (m64.abs() + spread)).all()
        assert ((rstd.double() - r64).abs() <= c * U * r64).all()
        bound = c * U * size + (2.0 ** -8 * y64.abs() if dtype == torch.bfloat16 else 0)
        assert ((y.double() - y64).abs() <= bound).all()
        if pad:      # a destination with a row stride of its own; what lies between its rows stays
            full = torch.full((rows, cols + pad), 7.0, device="cuda", dtype=dtype)
            ctx.layer_norm(x, w, b, EPS, out=full[:, :cols])
            assert torch.equal(full[:, :cols], y) and (full[:, cols:] == 7).all()
    assert ctx.status() == 0


def test_forward_of_constant_and_far_off_rows(ctx):
    # a constant row: xhat = 0, y = bias exactly, rstd = eps^-1/2; a mean 1e4 times the spread loses no more
    # than the bound above, which is relative to the spread
    cols = 1024
    w, b = params(cols, 1, 3)
    x = torch.full((3, cols), 3.0, device="cuda")
    y, mean, rstd = ctx.layer_norm(x, w, b, EPS)
    assert torch.equal(y, b.expand(3, cols)) and (mean == 3).all()
    assert ((rstd.double() - EPS ** -0.5).abs() <= 8 * U * EPS ** -0.5).all()
    far = make(5, cols, torch.float32, 3, mean=2e4)
    y, _, _ = ctx.layer_norm(far, w, b, EPS)
    y64, _, _, size, _ = norm64(far, w, b)
    assert ((y.double() - y64).abs() <= (32 + cols / 32) * U * size).all()


def test_rows_with_inf_and_nan_stay_apart(ctx):
    x = make(6, 300, torch.float32, 5)
    clean, _, _ = ctx.layer_norm(x, None, None, EPS)
    x = x.clone()
    x[1, 7] = float("inf")
    x[3, 299] = float("nan")
    x[4, 0] = -float("inf")
    y, _, _ = ctx.layer_norm(x, None, None, EPS)
    for r in (0, 2, 5):
        assert torch.equal(y[r], clean[r])
    for r in (1, 3, 4):
        assert torch.isnan(y[r]).all()


def bwd64(x, dy, mean, rstd, w):
    x, dy = x.double(), dy.double()
    w = torch.ones_like(x[0]) if w is None else w.double()
    r = rstd.double()[:, None]
    xhat = (x - mean.double()[:, None]) * r
    g = dy * w
    a, b = g.mean(1, keepdim=True), (g * xhat).mean(1, keepdim=True)
    dx = r * (g - a - xhat * b)
    size = r * (g.abs() + g.abs().mean(1, keepdim=True) + xhat.abs() * (g * xhat).abs().mean(1, keepdim=True))
    return dx, (dy * xhat).sum(0), dy.sum(0), size, (dy * xhat).abs().sum(0), dy.abs().sum(0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_backward(ctx, rows, cols, dtype):
    for pad, shift, which in ((0, 0, 1), (5, 0, 1), (8, 0, 0), (0, 1, 1)):
        x = make(rows, cols, dtype, rows + 7 * cols + pad, pad, shift)
        dy = make(rows, cols, dtype, rows + 9 * cols + pad, pad, shift, mean=0.1)
        w, _ = params(cols, cols, which)
        _, mean, rstd = ctx.layer_norm(x, w, None, EPS)
        dx, dw, db = ctx.layer_norm_bwd(dy, x, mean, rstd, w)
        dx64, dw64, db64, size, dw_size, db_size = bwd64(x, dy, mean, rstd, w)
        c = 32 + cols / 32
        bound = c * U * size + (2.0 ** -8 * dx64.abs() if dtype == torch.bfloat16 else 0)
        assert ((dx.double() - dx64).abs() <= bound).all()
        # sums over rows: at most `rows` sequential additions
        assert ((dw.double() - dw64).abs() <= (16 + rows) * U * dw_size).all()
        assert ((db.double() - db64).abs() <= (16 + rows) * U * db_size).all()
        # only what is asked for, with the same bits
        again = ctx.layer_norm_bwd(dy, x, mean, rstd, w, need_dweight=False, need_dbias=False)
        assert again[1] is None and again[2] is None and torch.equal(again[0], dx)
        again = ctx.layer_norm_bwd(dy, x, mean, rstd, w, need_dx=False)
        assert again[0] is None and torch.equal(again[1], dw) and torch.equal(again[2], db)
    assert ctx.status() == 0


def test_backward_against_differences(ctx):
    # central differences of the 64-bit forward form: h = 1e-5 leaves h^2-sized truncation and 1e-11-sized rounding
    rows, cols, h = 3, 37, 1e-5
    x, dy = make(rows, cols, torch.float32, 11), make(rows, cols, torch.float32, 12)
    w, b = params(cols, 13, 3)
    _, mean, rstd = ctx.layer_norm(x, w, b, EPS)
    dx, dw, db = ctx.layer_norm_bwd(dy, x, mean, rstd, w)

    def loss(x64, w64, b64):
        return (norm64(x64, w64, b64)[0] * dy.double()).sum().item()

    x64, w64, b64 = x.double(), w.double(), b.double()
    _, _, _, size, dw_size, db_size = bwd64(x, dy, mean, rstd, w)
    for r in range(rows):
        for c in range(cols):
            e = torch.zeros_like(x64)
            e[r, c] = h
            d = (loss(x64 + e, w64, b64) - loss(x64 - e, w64, b64)) / (2 * h)
            # 64 u covers the kernel and the binary32 mean and rstd it was given
            assert abs(dx[r, c].item() - d) <= 64 * U * (size[r].max().item() + 1) + 1e-8
    for c in range(cols):
        e = torch.zeros_like(w64)
        e[c] = h
        d = (loss(x64, w64 + e, b64) - loss(x64, w64 - e, b64)) / (2 * h)
        assert abs(dw[c].item() - d) <= 64 * U * (dw_size[c].item() + 1) + 1e-8
        d = (loss(x64, w64, b64 + e) - loss(x64, w64, b64 - e)) / (2 * h)
        assert abs(db[c].item() - d) <= 64 * U * (db_size[c].item() + 1) + 1e-8


def test_backward_repeats_bit_for_bit_and_takes_broadcast_gradients(ctx):
    x = make(3001, 520, torch.bfloat16, 21)
    w, _ = params(520, 3, 1)
    _, mean, rstd = ctx.layer_norm(x, w, None, EPS)
    dy = torch.ones(1, 1, device="cuda", dtype=torch.bfloat16).expand(3001, 520)     # the gradient of sum()
    first = ctx.layer_norm_bwd(dy, x, mean, rstd, w)
    full = ctx.layer_norm_bwd(dy.contiguous(), x, mean, rstd, w)
    for _ in range(20):
        again = ctx.layer_norm_bwd(dy, x, mean, rstd, w)
        assert all(torch.equal(a, b) for a, b in zip(first, again))
    assert all(torch.equal(a, b) for a, b in zip(first, full))
    assert (first[2] == 3001).all()


def test_no_rows(ctx):
    x = torch.empty(0, 64, device="cuda")
    y, mean, rstd = ctx.layer_norm(x)
    assert y.shape == (0, 64) and mean.numel() == 0
    dx, dw, db = ctx.layer_norm_bwd(x, x, mean, rstd)
    assert dx.shape == (0, 64) and not dw.any() and not db.any()
    q, s = ctx.quant_int8_rows(x)
    assert q.shape == (0, 64) and s.numel() == 0


def test_more_than_2_to_31_elements(ctx):
    rows, cols = 530_000, 4096
    x = torch.empty(rows, cols, device="cuda", dtype=torch.bfloat16)
    tail = make(64, cols, torch.bfloat16, 9)
    x[:64] = tail
    x[64:-64] = 1
    x[-64:] = tail
    y, mean, rstd = ctx.layer_norm(x, None, None, EPS)
    assert torch.equal(y[-64:], y[:64]) and torch.equal(mean[-64:], mean[:64])
    q, s = ctx.quant_int8_rows(x)
    assert torch.equal(q[-64:], q[:64]) and torch.equal(s[-64:], s[:64])
    del q, s
    dx, dw, db = ctx.layer_norm_bwd(y, x, mean, rstd)
    assert torch.equal(dx[-64:], dx[:64])
    torch.cuda.synchronize()
    assert ctx.status() == 0


# ---- int8 rows -----------------------------------------------------------------------------------------------

def codes32(x):
    """The definition, in binary32 with numpy: scale = max / 127, q = rint(x * (127 * (1 / max)))."""
    x = x.float().cpu().numpy()
    top = np.abs(x).max(1)
    with np.errstate(divide="ignore"):
        factor = np.where(top > 0, np.float32(127) * (np.float32(1) / top), np.float32(0)).astype(np.float32)
    return np.rint(x * factor[:, None]).astype(np.int8), (top / np.float32(127)).astype(np.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_codes_are_the_definitions(ctx, rows, cols, dtype):
    for pad, shift in ((0, 0), (5, 0), (8, 0), (0, 1)):
        x = make(rows, cols, dtype, rows + cols + pad, pad, shift)
        if rows > 2:
            x = x.clone() if pad == 0 and shift == 0 else x
            x[1] = 0
        q, s = ctx.quant_int8_rows(x)
        q32, s32 = codes32(x)
        assert np.array_equal(q.cpu().numpy(), q32) and np.array_equal(s.cpu().numpy(), s32)
        assert q.stride(0) % 16 == 0 or rows == 1
    assert ctx.status() == 0


def test_ties_go_to_even_and_zero_rows_stay_zero(ctx):
    x = torch.zeros(2, 16, device="cuda")
    x[0, :5] = torch.tensor([127.0, 0.5, 1.5, 2.5, -3.5], device="cuda")
    q, s = ctx.quant_int8_rows(x)
    assert q[0, :5].tolist() == [127, 0, 2, 2, -4] and s.tolist() == [1.0, 0.0] and not q[1].any()


@pytest.mark.parametrize("cols", [5, 64, 1000, 4096, 40000])
def test_rows_that_cannot_be_scaled(ctx, cols):
    x = make(5, cols, torch.float32, 3).clone()
    x[0, 1] = float("inf")
    x[2] = 2.0 ** -101
    x[3, cols - 1] = float("nan")
    q, s = ctx.quant_int8_rows(x)
    assert ctx.status() == binding.STATUS_NONFINITE | binding.STATUS_RANGE
    assert not q[0].any() and not q[2].any() and not q[3].any()
    assert torch.isnan(s[0]) and s[2] == 0 and torch.isnan(s[3])
    keep = [1, 4]
    q2, s2 = ctx.quant_int8_rows(x[keep].contiguous())
    assert torch.equal(q[keep], q2) and torch.equal(s[keep], s2)
    assert ctx.status() == 0


def test_the_largest_numbers_are_scaled(ctx):
    x = torch.tensor([[3.4e38, -1.7e38, 0.0, 1.0], [2.0 ** -100, -2.0 ** -101, 0, 0]], device="cuda")
    q, s = ctx.quant_int8_rows(x)
    q32, s32 = codes32(x)
    assert np.array_equal(q.cpu().numpy(), q32) and np.array_equal(s.cpu().numpy(), s32)
    assert ctx.status() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norm_to_codes(ctx, rows, cols, dtype):
    for pad, shift, which in ((0, 0, 3), (5, 0, 0), (8, 1, 3)):
        x = make(rows, cols, dtype, rows + 3 * cols + pad, pad, shift)
        w, b = params(cols, cols, which)
        q, s = ctx.layer_norm_int8(x, w, b, EPS)
        y64, _, _, size, _ = norm64(x, w, b)
        err = (32 + cols / 32) * U * size            # of the value that is quantized
        s64 = y64.abs().amax(1) / 127
        assert ((s.double() - s64).abs() <= err.amax(1) / 127 + 2 * U * s64).all()
        # half a step, what the value itself is off, and the rounding of factor and product (4 u of 127 steps)
        off = (q.double() * s.double()[:, None] - y64).abs()
        assert (off <= (0.5 + 4 * 127 * U) * s.double()[:, None] + 2 * err).all()
    # one-element rows: a layer norm of one value is its bias (or zero)
    assert ctx.status() == 0


def test_refusals(ctx):
    x = make(4, 64, torch.float32, 1)
    _, mean, rstd = ctx.layer_norm(x)
    with pytest.raises(TypeError):
        ctx.layer_norm(x.half())
    with pytest.raises(TypeError):
        ctx.layer_norm(x, torch.ones(63, device="cuda"))
    with pytest.raises(TypeError):
        ctx.layer_norm(x, torch.ones(64, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        ctx.layer_norm(x.cpu())
    with pytest.raises(TypeError):
        ctx.layer_norm(x, out=torch.empty(4, 64, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        ctx.layer_norm(x, out=torch.empty(3, 64, device="cuda"))
    with pytest.raises(binding.LuqError) as e:
        ctx.layer_norm(x, eps=float("nan"))
    assert e.value.code == binding.ERR_ARG
    with pytest.raises(binding.LuqError):
        ctx.layer_norm(torch.empty(4, 0, device="cuda"))
    with pytest.raises(TypeError):
        ctx.layer_norm_bwd(x.bfloat16(), x, mean, rstd)
    with pytest.raises(TypeError):
        ctx.layer_norm_bwd(x, x, mean[:3], rstd)
    with pytest.raises(binding.LuqError):
        ctx.quant_int8_rows(torch.empty(4, 0, device="cuda"))
    L, s = binding.load(), torch.cuda.current_stream().cuda_stream
    q = torch.empty(4, 64, device="cuda", dtype=torch.int8)
    p = x.data_ptr()
    rows8 = lambda **k: L.luq_quant_int8_rows(ctx.handle, k.get("x", p), k.get("dtype", 0), k.get("rows", 4), 64,  # noqa: E731
                                              k.get("ld", 64), q.data_ptr() + k.get("off", 0), k.get("ldq", 64), mean.data_ptr(), s)
    assert rows8() == 0
    for bad in ({"x": None}, {"x": p + 2}, {"dtype": 2}, {"rows": -1}, {"ld": 63}, {"off": 8}, {"ldq": 72}, {"ldq": 48}):
        assert rows8(**bad) == binding.ERR_ARG, bad
    assert ctx.status() == 0
