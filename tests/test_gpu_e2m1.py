"""Microscaled 4-bit floating point: quantizer and products against the definition in 64 bits.

Tolerances.  Codes and scales are exact.  A product's sums are binary32: each of the at most K / 16 + 12 additions and products that
make an output (blocks, parts of a split contraction, scales, bias) may be off by one step, 2^-23, of the sum of magnitudes; a bf16
output by half of one more step of its own, 2^-8."""
import pytest
import torch

from paper_2112_10769_b200 import binding, e2m1

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def tokens(rows, cols, dtype=torch.float32, seed=0, pad=0, shift=0):
    """Rows of different size with channels far above the others, cut out of a wider tensor."""
    g = torch.Generator("cuda").manual_seed(1000 * rows + cols + seed)
    x = torch.randn(rows * (cols + pad) + shift, device="cuda", generator=g)
    x = x[shift:].view(rows, cols + pad)
    x *= torch.exp(torch.randn(rows, 1, device="cuda", generator=g))
    x[:, ::17] *= 8
    base = torch.zeros(rows * (cols + pad) + shift, dtype=dtype, device="cuda")
    base[shift:] = x.to(dtype).flatten()
    return base[shift:].view(rows, cols + pad)[:, :cols]


def rounded(v):
    """e2m1 by the borders between its numbers; a border goes to the even code."""
    a, out = v.abs(), torch.zeros_like(v)
    for border, up, level in ((0.25, False, 0.5), (0.75, True, 1.0), (1.25, False, 1.5), (1.75, True, 2.0), (2.5, False, 3.0), (3.5, True, 4.0), (5.0, False, 6.0)):
        out = torch.where(a >= border if up else a > border, torch.full_like(out, level), out)
    return out * torch.sign(v)


def definition(x, block):
    """The values that the quantized rows stand for; quotients and products of two binary32 numbers, rounded to binary32 from 64 bits,
    are the binary32 ones."""
    f32 = lambda v: v.float().double()
    rows, cols = x.shape
    full = torch.zeros(rows, -(-cols // block) * block, dtype=torch.float64, device=x.device)
    full[:, :cols] = x.double()
    b = full.unflatten(1, (-1, block))
    top = b.abs().amax(2, keepdim=True)
    if block == 32:
        s = torch.exp2(((top.float().view(torch.int32) >> 23) - 129).clamp_min(-127).double())
        return (rounded(b / s) * s).flatten(1)[:, :cols]
    row = top.amax(1, keepdim=True)
    g = torch.where(row >= 2.0 ** -100, f32(row / 2688), 0.0)
    s = torch.where(g > 0, f32(top / f32(6 * torch.where(g > 0, g, 1.0))), 0.0).float().to(torch.float8_e4m3fn).double()
    r = torch.where(s > 0, f32(1 / torch.where(s > 0, f32(s * g), 1.0)), 0.0)
    return (rounded(f32(b * r)) * s * g).flatten(1)[:, :cols]


def close(z, want, mag, K):
    # (where nothing was summed, nothing may be off)
    bound = (K / 16 + 12) * 2.0 ** -23 * mag
    if z.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (want.abs() + bound)
    assert ((z.double() - want).abs() <= bound).all()


# widths of one element, of part of a block, of a tile, odd ones, one for every path of the kernel up to rows that are read twice
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,pad,shift", [(1, 1, 0, 0), (3, 15, 0, 0), (5, 16, 0, 0), (130, 33, 3, 1), (7, 64, 0, 0), (300, 100, 0, 3), (129, 257, 0, 0),
                                                 (2, 512, 8, 0), (700, 511, 0, 0), (601, 1000, 0, 0), (700, 1024, 0, 0), (3, 1023, 2, 5), (650, 2000, 0, 0), (2, 4096, 0, 0),
                                                 (4, 4097, 0, 0), (700, 4097, 1, 1), (3, 16384, 0, 0), (620, 9000, 0, 0), (2, 32768, 0, 0), (2, 33001, 0, 0)])
def test_quantizer(ctx, rows, cols, pad, shift, dtype, block):
    x = tokens(rows, cols, dtype, 0, pad, shift)
    codes, tiles, scale = ctx.quant_e2m1_rows(x, block)
    assert codes.shape == (rows, -(-cols // 2)) and (scale is None) == (block == 32)
    assert torch.equal(e2m1.values(codes, tiles, scale, cols, block), definition(x, block))
    if cols % 2:
        assert (codes[:, -1] >> 4 == 0).all()
    # blocks beyond the row's end have zero scales
    beyond = e2m1.scale_rows(tiles, rows, tiles.shape[1] * 4 * block, block)[:, -(-cols // block):]
    assert (beyond == 0).all() and ctx.status() == 0


# so many rows that a thread takes several pieces of each: rows of a warp and of a block, whole and ragged, aligned and not
MANY = [(4801, 2000, 0, 0), (9500, 1041, 1, 1), (5000, 1025, 7, 0), (18500, 2065, 0, 0), (9500, 4096, 0, 0), (9500, 4097, 1, 3), (2400, 16384, 0, 0)]


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("rows,cols,pad,shift", MANY)
def test_quantizer_of_many_rows(ctx, rows, cols, pad, shift, block):
    x = tokens(rows, cols, torch.bfloat16, 0, pad, shift)
    x[rows // 2, cols // 3] = 0.0
    x[rows - 1] = 0.0
    codes, tiles, scale = ctx.quant_e2m1_rows(x, block)
    assert torch.equal(e2m1.values(codes, tiles, scale, cols, block), definition(x, block))
    beyond = e2m1.scale_rows(tiles, rows, tiles.shape[1] * 4 * block, block)[:, -(-cols // block):]
    assert (beyond == 0).all() and ctx.status() == 0
    x[7, cols - 1], x[rows - 2, 0] = NAN, INF                 # two rows of neither numbers nor a scale leave the others as they are
    again, tiles2, scale2 = ctx.quant_e2m1_rows(x, block)
    others = torch.ones(rows, dtype=torch.bool, device="cuda")
    others[7] = others[rows - 2] = False
    assert torch.equal(again[others], codes[others]) and ctx.status() == binding.STATUS_NONFINITE
    a, b = e2m1.scale_rows(tiles, rows, cols, block), e2m1.scale_rows(tiles2, rows, cols, block)
    assert torch.equal(a[others].view(torch.uint8), b[others].view(torch.uint8))


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("rows,cols,pad,shift", [(5000, 1999, 1, 0), (9500, 4096, 0, 0)])
def test_quantizer_of_many_copies(ctx, rows, cols, pad, shift, block):
    x = tokens(rows, cols, torch.bfloat16, 0, pad, shift)
    g = torch.Generator("cuda").manual_seed(rows)
    chosen = torch.rand(rows, 7, device="cuda", generator=g).topk(2, dim=1).indices.int()
    chosen[::5, 1] = -1
    offsets, position = ctx.expert_order(chosen, 7)
    codes, tiles, scale = ctx.quant_e2m1_rows(x, block)
    at, tiles_at, scale_at = ctx.quant_e2m1_rows(x, block, offsets=offsets, position=position)
    there = position >= 0
    token = torch.arange(rows, device="cuda")[:, None].expand(-1, 2)[there]
    to = position[there].long()
    assert torch.equal(at[to], codes[token])
    if block == 16:
        assert torch.equal(scale_at[to], scale[token])
    plain = e2m1.scale_rows(tiles, rows, cols, block).view(torch.uint8)
    source = torch.empty(int(there.sum()), dtype=torch.long, device="cuda")
    source[to] = token
    ends = offsets.tolist()
    for e in range(7):
        n = ends[e + 1] - ends[e]
        got = e2m1.scale_rows(tiles_at[ends[e] // 128 + e:], n, cols, block).view(torch.uint8)
        assert torch.equal(got, plain[source[ends[e]:ends[e + 1]]])
    assert ctx.status() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantizer_at_the_borders(ctx, dtype):
    # every border between two numbers, and the patterns next to it, with scales that are powers of two; the first element is the largest
    borders = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=dtype, device="cuda")
    x = torch.zeros(6, 64, dtype=dtype, device="cuda")
    bits = borders.view(torch.int32 if dtype == torch.float32 else torch.int16)
    for r, (off, sign) in enumerate([(0, 1), (1, 1), (-1, 1), (0, -1), (1, -1), (-1, -1)]):
        x[r, 0], x[r, 32] = 6.0, 6.0
        x[r, 1:8] = sign * (bits + off).view(dtype)
        x[r, 33:40] = x[r, 1:8] * 2.0 ** -6 if r % 2 else x[r, 1:8]
    for block in (16, 32):
        codes, tiles, scale = ctx.quant_e2m1_rows(x, block)
        assert torch.equal(e2m1.values(codes, tiles, scale, 64, block), definition(x, block))


def test_quantizer_of_rows_without_a_scale(ctx):
    x = torch.zeros(12, 96, device="cuda")
    x[1, 5] = 1e-31                                          # below 2^-100
    x[2, 5], x[2, 40] = 3e38, -1.0                           # the second block is nothing beside the first
    x[3] = torch.finfo(torch.float32).tiny
    x[4, 7], x[4, 50] = 1e-42, 1e-45                         # subnormal
    x[5, 9], x[5, 70] = INF, 1.0
    x[6, 9], x[6, 70] = NAN, 1.0
    x[7, 95] = -INF
    x[8] = 1.0
    x[9, 0], x[9, 40] = 448.0 * 6, 2.0 ** -10 * 6            # the smallest e4m3 scale
    x[10, 0], x[10, 40] = 448.0 * 6, 2.0 ** -10 * 6 * 0.49   # less than half of it: a zero scale
    finite = [0, 1, 2, 3, 4, 8, 9, 10, 11]
    for block in (16, 32):
        for rows, flags in ((finite, binding.STATUS_RANGE if block == 16 else 0), ([0, 5, 6, 7, 8], binding.STATUS_NONFINITE)):
            codes, tiles, scale = ctx.quant_e2m1_rows(x[rows], block)
            assert ctx.status() == flags
            v = e2m1.values(codes, tiles, scale, 96, block)
            if rows is finite:
                assert torch.equal(v, definition(x[rows], block))
            else:
                bad = torch.isnan(v)
                assert bad[1:4].any(1).all() and not bad[0].any() and not bad[4].any()
                assert torch.equal(v[4], definition(x[8:9], block)[0])
                # in a product: NaN for the row, numbers for the others
                w = e2m1.quantize_weight(torch.ones(40, 96, device="cuda"), block)
                z = ctx.gemm_e2m1(codes, tiles, scale, *w, block=block)
                assert torch.isnan(z[1:4]).all() and torch.isfinite(z[[0, 4]]).all()


def test_quantizer_of_several_matrices(ctx):
    w = torch.randn(3, 130, 200, device="cuda")
    for block in (16, 32):
        codes, tiles, scale = e2m1.quantize_weight(w, block)
        assert codes.shape == (3, 130, 100)
        for e in range(3):
            c, t, s = ctx.quant_e2m1_rows(w[e], block)
            assert torch.equal(codes[e], c) and torch.equal(e2m1.values(codes[e], tiles[2 * e:2 * e + 2], None if s is None else scale[e], 200, block),
                                                            e2m1.values(c, t, s, 200, block))
    codes, tiles, scale = e2m1.quantize_weight(w.view(3, 2, 65, 200))
    assert codes.shape == (3, 2, 65, 100) and scale.shape == (3, 2, 65) and tiles.shape[0] == 6


SIZES = [(1, 1, 1), (1, 128, 64), (2, 100, 37), (5, 129, 300), (31, 64, 4096), (33, 300, 512), (64, 257, 65), (65, 128, 1000), (100, 1000, 129), (129, 130, 2000),
         (200, 520, 256), (300, 4097, 100), (333, 1537, 1000), (514, 300, 4100), (1000, 256, 640), (2500, 700, 300), (5000, 2050, 520), (1, 70, 70001)]


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_product(ctx, M, N, K, block):
    dtype = torch.bfloat16 if (M + N) % 2 else torch.float32
    x, w, bias = tokens(M, K, dtype), tokens(N, K, torch.float32, 1), torch.randn(N, device="cuda")
    q, wq = ctx.quant_e2m1_rows(x, block), e2m1.quantize_weight(w, block)
    xv, wv = e2m1.values(*q, K, block), e2m1.values(*wq, K, block)
    want, mag = xv @ wv.t() + bias.double(), xv.abs() @ wv.abs().t() + bias.abs().double()
    for out_dtype in (torch.float32, torch.bfloat16):
        z = ctx.gemm_e2m1(*q, *wq, bias, block, out_dtype=out_dtype)
        close(z, want, mag, K)
        # one call is the two calls bit for bit, and a call repeats
        assert torch.equal(ctx.quant_e2m1_gemm(x, *wq, bias, block, out_dtype=out_dtype), z)
        assert torch.equal(ctx.gemm_e2m1(*q, *wq, bias, block, out_dtype=out_dtype), z)
    close(ctx.gemm_e2m1(*q, *wq, None, block), want - bias.double(), mag, K)
    assert ctx.status() == 0


@pytest.mark.parametrize("pad,shift", [(0, 0), (1, 0), (8, 0), (4, 1), (3, 3)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_product_into_a_part_of_a_tensor(ctx, dtype, pad, shift):
    for M, N, K in ((3, 100, 64), (70, 131, 300), (1000, 520, 260), (700, 1001, 64)):
        x, w = tokens(M, K), tokens(N, K, torch.float32, 1)
        wq = e2m1.quantize_weight(w)
        base = torch.full((shift + M * (N + pad) + 5,), 7.0, dtype=dtype, device="cuda")
        out = base[shift:shift + M * (N + pad)].view(M, N + pad)
        ctx.quant_e2m1_gemm(x, *wq, out=out[:, :N])
        assert torch.equal(out[:, :N], ctx.quant_e2m1_gemm(x, *wq, out_dtype=dtype))
        assert (out[:, N:] == 7).all() and (base[:shift] == 7).all() and (base[shift + M * (N + pad):] == 7).all()


def test_rows_beyond_32_bits(ctx):
    # 2.6e9 elements in, 2.3e9 out: a row's answer does not depend on where it lies (the same tiles, the same sums)
    M, N, K = 320000, 7200, 8192
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    part = tokens(256, K, torch.bfloat16)
    wq = e2m1.quantize_weight(tokens(N, K, torch.float32, 1))
    first = M - 512                                            # (a tile's first row)
    x[first:first + 256] = part
    z = ctx.quant_e2m1_gemm(x, *wq)
    assert (z[:first] == 0).all() and (z[first + 256:] == 0).all()
    q = ctx.quant_e2m1_rows(part)
    xv, wv = e2m1.values(*q, K), e2m1.values(*wq, K)
    close(z[first:first + 256], xv @ wv.t(), xv.abs() @ wv.abs().t(), K)


def test_scales_from_elsewhere(ctx):
    # any e4m3 scales and any row scales, negative ones among them, and codes in rows further apart
    g = torch.Generator("cuda").manual_seed(1)
    M, N, K = 70, 140, 320
    def matrix(rows):
        codes = torch.randint(0, 256, (rows, K // 2 + 48), dtype=torch.uint8, device="cuda", generator=g)[:, :K // 2]
        s = torch.randn(rows, K // 16, device="cuda", generator=g).to(torch.float8_e4m3fn)
        return codes, e2m1.scale_tiles(s, 16), torch.randn(rows, device="cuda", generator=g)
    x, w = matrix(M), matrix(N)
    s32 = lambda rows: e2m1.scale_tiles(torch.randint(100, 150, (rows, K // 32), dtype=torch.uint8, device="cuda", generator=g), 32)
    for block, a, b in ((16, x, w), (32, (x[0], s32(M), None), (w[0], s32(N), None))):
        xv, wv = e2m1.values(*a, K, block), e2m1.values(*b, K, block)
        close(ctx.gemm_e2m1(*a, *b, block=block), xv @ wv.t(), xv.abs() @ wv.abs().t(), K)


def grouped_case(E, N, K, ends, block, dtype, seed=0):
    M = 1 + max(ends)
    x, w = tokens(M, K, dtype, seed), torch.randn(E, N, K, device="cuda")
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    return M, x, e2m1.quantize_weight(w, block), torch.randn(E, N, device="cuda"), offsets


# empty groups, groups of one row, that end in a tile of scales and at its end, many; rows before the first and behind the last
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("N,K,ends", [(100, 64, [0, 5]), (130, 300, [0, 0, 1, 1, 40, 40]), (64, 512, [3, 130, 131, 259, 700]), (300, 100, [0, 128, 256, 256, 1000, 1001]),
                                      (40, 1000, [0, 1, 2, 3, 4, 5, 6, 7, 8]), (520, 640, [10, 1400, 1500, 3000]), (72, 96, list(range(0, 2000, 17)))])
def test_grouped(ctx, N, K, ends, block):
    E = len(ends) - 1
    dtype = torch.float32 if N % 3 else torch.bfloat16
    M, x, wq, bias, offsets = grouped_case(E, N, K, ends, block, dtype)
    out = torch.full((M, N), 5.0, dtype=dtype, device="cuda")
    ctx.quant_e2m1_gemm_grouped(x, offsets, *wq, bias, block, out=out)
    q = ctx.quant_e2m1_rows(x, block, offsets=offsets)
    again = torch.full((M, N), 5.0, dtype=dtype, device="cuda")
    assert torch.equal(ctx.gemm_e2m1_grouped(*q, offsets, *wq, bias, block, out=again), out)
    assert (out[:ends[0]] == 5).all() and (out[ends[-1]:] == 5).all() and ctx.status() == 0
    tiles = wq[1].shape[0] // E
    for e in range(E):
        a, b = ends[e], ends[e + 1]
        if a < b:
            we = (wq[0][e], wq[1][e * tiles:(e + 1) * tiles], None if block == 32 else wq[2][e])
            xv, wv = definition(x[a:b], block), e2m1.values(*we, K, block)
            close(out[a:b], xv @ wv.t() + bias[e].double(), xv.abs() @ wv.abs().t() + bias[e].abs().double(), K)


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("T,k,E,N,K", [(1, 1, 1, 40, 64), (1, 8, 64, 200, 300), (48, 2, 16, 128, 1000), (700, 3, 5, 260, 130), (3000, 2, 300, 64, 64)])
def test_grouped_by_positions(ctx, T, k, E, N, K, block):
    g = torch.Generator("cuda").manual_seed(T)
    x = tokens(T, K, torch.bfloat16)
    wq, bias = e2m1.quantize_weight(torch.randn(E, N, K, device="cuda"), block), torch.randn(E, N, device="cuda")
    chosen = torch.rand(T, E, device="cuda", generator=g).topk(min(k, E), 1).indices.to(torch.int32)
    chosen[T // 2:T // 2 + T // 10] = -1
    offsets, position = ctx.expert_order(chosen, E)
    out = torch.full((position.numel(), N), 5.0, dtype=torch.bfloat16, device="cuda")
    ctx.quant_e2m1_gemm_grouped(x, offsets, *wq, bias, block, position=position, out=out)
    # the same as copying the tokens first
    rows = ctx.dispatch(x, position, offsets)
    want = torch.full_like(out, 5.0)
    ctx.quant_e2m1_gemm_grouped(rows, offsets, *wq, bias, block, out=want)
    assert torch.equal(out, want) and (out[int(offsets[-1]):] == 5).all() and ctx.status() == 0


def test_offsets_that_are_none(ctx):
    # decreasing, negative, beyond the rows: flagged, and nothing outside the tensors is touched
    M, x, wq, bias, _ = grouped_case(4, 72, 128, [0, 100, 200, 300, 400], 16, torch.float32)
    for bad in ([0, 300, 200, 350, 400], [-5, 10, 20, 30, 40], [0, 10, 20, 30, 1 << 30], [400, 300, 200, 100, 0]):
        offsets = torch.tensor(bad, dtype=torch.int32, device="cuda")
        base = torch.full((M + 20, 72), 5.0, device="cuda")
        ctx.quant_e2m1_gemm_grouped(x, offsets, *wq, bias, out=base[10:10 + M])
        assert ctx.status() & binding.STATUS_OFFSETS
        assert (base[:10] == 5).all() and (base[10 + M:] == 5).all()
    # positions that are none are left out
    position = torch.full((M, 1), -1, dtype=torch.int32, device="cuda")
    position[:3, 0] = torch.tensor([0, 1 << 30, -(1 << 30)], dtype=torch.int32)
    offsets = torch.tensor([0, 1, 1, 1, 1], dtype=torch.int32, device="cuda")
    z = ctx.quant_e2m1_gemm_grouped(x, offsets, *wq, bias, position=position)
    assert torch.equal(z[:1], ctx.quant_e2m1_gemm_grouped(x[:1].contiguous(), offsets, *wq, bias)) and ctx.status() == 0


def test_nothing_to_do(ctx):
    wq = e2m1.quantize_weight(torch.randn(40, 64, device="cuda"))
    assert ctx.quant_e2m1_gemm(torch.empty(0, 64, device="cuda"), *wq).shape == (0, 40)
    codes, tiles, scale = ctx.quant_e2m1_rows(torch.empty(0, 64, device="cuda"))
    assert codes.shape == (0, 32) and tiles.numel() == 0 and scale.numel() == 0
    we = e2m1.quantize_weight(torch.randn(3, 40, 64, device="cuda"))
    offsets = torch.zeros(4, dtype=torch.int32, device="cuda")
    assert ctx.quant_e2m1_gemm_grouped(torch.empty(0, 64, device="cuda"), offsets, *we).shape == (0, 40)
    assert ctx.status() == 0


def test_refusals(ctx):
    x = tokens(8, 64)
    wq = e2m1.quantize_weight(torch.randn(40, 64, device="cuda"))
    we = e2m1.quantize_weight(torch.randn(3, 40, 64, device="cuda"))
    offsets = torch.tensor([0, 2, 4, 8], dtype=torch.int32, device="cuda")
    q = ctx.quant_e2m1_rows(x)
    shifted = torch.zeros(41 * 32 + 1, dtype=torch.uint8, device="cuda")[1:40 * 32 + 1].view(40, 32)
    for call in (lambda: ctx.quant_e2m1_rows(x, 8), lambda: ctx.quant_e2m1_rows(x.half()), lambda: ctx.quant_e2m1_rows(x, planes=3),
                 lambda: ctx.quant_e2m1_rows(x, position=torch.zeros(8, 1, dtype=torch.int32, device="cuda")),
                 lambda: ctx.quant_e2m1_rows(x, offsets=offsets.long()), lambda: ctx.quant_e2m1_rows(x, planes=2, offsets=offsets),
                 lambda: ctx.quant_e2m1_gemm(x[:, :32], *wq), lambda: ctx.quant_e2m1_gemm(x, wq[0], wq[1], None),
                 lambda: ctx.quant_e2m1_gemm(x, *wq, block=32), lambda: ctx.quant_e2m1_gemm(x, wq[0], wq[1][:, :, :256], wq[2]),
                 lambda: ctx.quant_e2m1_gemm(x, wq[0], wq[1], wq[2][:3]), lambda: ctx.quant_e2m1_gemm(x, shifted, wq[1], wq[2]),
                 lambda: ctx.quant_e2m1_gemm(x, wq[0].to(torch.int8), wq[1], wq[2]), lambda: ctx.quant_e2m1_gemm(x.cpu(), *wq),
                 lambda: ctx.quant_e2m1_gemm(x, *wq, torch.zeros(39, device="cuda")), lambda: ctx.quant_e2m1_gemm(x, *wq, out=torch.empty(8, 41, device="cuda")),
                 lambda: ctx.gemm_e2m1(q[0], q[1], None, *wq), lambda: ctx.gemm_e2m1(q[0][:, :16], q[1], q[2], *wq),
                 lambda: ctx.quant_e2m1_gemm_grouped(x, offsets[:3], *we), lambda: ctx.quant_e2m1_gemm_grouped(x, offsets, *wq),
                 lambda: ctx.quant_e2m1_gemm_grouped(x, offsets, *we, position=torch.zeros(7, 2, dtype=torch.int32, device="cuda")),
                 lambda: ctx.quant_e2m1_gemm_grouped(x, offsets, *we, position=torch.zeros(8, dtype=torch.int32, device="cuda")),
                 lambda: ctx.gemm_e2m1_grouped(*q, offsets, *we)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        e2m1.E2m1Linear(torch.randn(3, 40, 64, device="cuda"))
    with pytest.raises(ValueError):
        e2m1.E2m1Experts(torch.randn(40, 64, device="cuda"))
    assert ctx.status() == 0


def test_limited_to_some_multiprocessors(ctx):
    x, w = tokens(300, 1000, torch.bfloat16), torch.randn(700, 1000, device="cuda")
    wq = e2m1.quantize_weight(w)
    xv, wv = definition(x, 16), e2m1.values(*wq, 1000)
    for limit in (1, 2, 7, 0):
        ctx.set_option(binding.OPT_SM_LIMIT, limit)
        for M in (1, 2, 40, 300):
            close(ctx.quant_e2m1_gemm(x[:M], *wq), xv[:M] @ wv.t(), xv[:M].abs() @ wv.abs().t(), 1000)
    assert ctx.status() == 0


def test_modules(ctx):
    torch.manual_seed(0)
    x = tokens(30, 200, torch.bfloat16)
    layer = torch.nn.Linear(200, 72, device="cuda")
    experts = torch.randn(4, 72, 200, device="cuda")
    for block in (16, 32):
        m = e2m1.E2m1Linear.of(layer, block)
        want = ctx.quant_e2m1_gemm(x, *e2m1.quantize_weight(layer.weight, block), layer.bias.detach(), block)
        assert torch.equal(m(x), want) and torch.equal(m(x.view(5, 6, 200)), want.view(5, 6, 72))
        # casting leaves what the kernels read as it is, a state dict brings it back
        state = {k: v.clone() for k, v in m.state_dict().items()}
        assert torch.equal(m.bfloat16()(x), want)
        other = e2m1.E2m1Linear(torch.zeros(72, 200, device="cuda"), torch.zeros(72, device="cuda"), block)
        other.load_state_dict(state)
        assert torch.equal(other(x), want)
        e = e2m1.E2m1Experts(experts, block=block)
        offsets = torch.tensor([0, 10, 10, 25, 30], dtype=torch.int32, device="cuda")
        assert torch.equal(e(x, offsets), ctx.quant_e2m1_gemm_grouped(x, offsets, *e2m1.quantize_weight(experts, block), block=block))
        for i, (a, b) in enumerate([(0, 10), (10, 10), (10, 25), (25, 30)]):
            if a < b:
                assert torch.equal(e(x, offsets)[a:b], e2m1.E2m1Linear(experts[i], block=block)(x[a:b]))
    # a token's answer does not depend on the others beside it, but for the order of its sums
    m = e2m1.E2m1Linear.of(layer)
    one = torch.cat([m(x[i:i + 1].float()) for i in range(30)])
    torch.testing.assert_close(one, m(x.float()), rtol=1e-5, atol=1e-4)


def test_graphs_and_streams(ctx):
    wq = e2m1.quantize_weight(torch.randn(500, 1000, device="cuda"))
    xs = [tokens(200, 1000, torch.bfloat16, s) for s in range(4)]
    want = [ctx.quant_e2m1_gemm(x, *wq) for x in xs]
    # two captured calls share no workspace: replayed side by side on two streams
    graphs = []
    for s in range(2):
        x, stream = xs[s].clone(), torch.cuda.Stream()
        with torch.cuda.stream(stream):
            ctx.quant_e2m1_gemm(x, *wq)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                z = ctx.quant_e2m1_gemm(x, *wq)
        graphs.append((g, x, z, stream))
    torch.cuda.synchronize()
    for turn in range(20):
        for g, x, z, stream in graphs:
            with torch.cuda.stream(stream):
                x.copy_(xs[(turn + (g is graphs[1][0])) % 4])
                g.replay()
        torch.cuda.synchronize()
        for i, (_, _, z, _) in enumerate(graphs):
            assert torch.equal(z, want[(turn + i) % 4])
    assert ctx.status() == 0
