"""int8 products with a scale for each token and output channel, plain and grouped by expert, against 64 bits.

Tolerance.  The integer sums are exact in int32; the sum's conversion to binary32, the product with the
channel's scale and the fused multiply-add with the token's scale and the bias are one rounding each, so
|z - z64| <= 2 u |z64 - bias| + u |z64| with u = 2^-24, to first order; asserted with 4 u (|z64 - bias| + |bias|).
bf16 results add one rounding, at most 2^-9 of the value (asserted with 2^-8)."""
import pytest
import torch

from paper_2112_10769_b200 import binding

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def codes(rows, cols, seed, ld=None, lead=()):
    g = torch.Generator("cuda").manual_seed(seed)
    ld = -(-cols // 16) * 16 if ld is None else ld
    return torch.randint(-127, 128, (*lead, rows, ld), device="cuda", dtype=torch.int8, generator=g)[..., :cols]


def floats(n, seed):
    return torch.rand(n, device="cuda", generator=torch.Generator("cuda").manual_seed(seed)) * 0.02 + 1e-3


def reference(x, sx, w, sw, bias):
    z = (x.double() @ w.double().t()) * sx.double()[:, None] * sw.double()
    return z if bias is None else z + bias.double()


def check(z, x, sx, w, sw, bias):
    ref = reference(x, sx, w, sw, bias)
    b = 0 if bias is None else bias.double()
    bound = 4 * U * ((ref - b).abs() + (0 if bias is None else b.abs()))
    if z.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * ref.abs()
    off = (z.double() - ref).abs()
    assert (off <= bound).all(), (off - bound).max().item()


SIZES = [(1, 1, 1), (1, 128, 128), (2, 3, 16), (1, 4096, 1024), (5, 127, 15), (8, 129, 17), (15, 31, 300), (16, 256, 128), (17, 130, 129),
         (31, 500, 1000), (32, 128, 256), (33, 257, 127), (63, 64, 640), (64, 512, 512), (65, 96, 2048), (100, 1000, 72),
         (127, 384, 128), (128, 128, 4096), (129, 513, 200), (256, 256, 256), (300, 72, 1111), (333, 1537, 1000),
         (511, 640, 384), (512, 1024, 64), (513, 200, 528), (777, 2000, 96), (1024, 512, 1024), (1025, 129, 130),
         (1300, 1100, 260), (2048, 2304, 512), (4100, 384, 96), (40000, 8, 16), (3, 40000, 64), (700, 300, 8192), (4, 64, 16384)]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_product(ctx, M, N, K):
    x, w = codes(M, K, M + N), codes(N, K, M + N + 1)
    sx, sw, bias = floats(M, 1), floats(N, 2), floats(N, 3) - 0.01
    for dtype in (torch.float32, torch.bfloat16):
        for b in (None, bias):
            check(ctx.gemm_int8(x, sx, w, sw, b, out_dtype=dtype), x, sx, w, sw, b)
    assert ctx.status() == 0


@pytest.mark.parametrize("M,N,K", [(1, 100, 48), (33, 257, 127), (130, 128, 300), (700, 520, 256), (1100, 1000, 130)])
def test_strides_and_alignment(ctx, M, N, K):
    x, w = codes(M, K, 5, ld=-(-K // 16) * 16 + 48), codes(N, K, 6, ld=-(-K // 16) * 16 + 16)
    sx, sw, bias = floats(M, 1), floats(N, 2), floats(N, 3)
    for dtype in (torch.float32, torch.bfloat16):
        want = ctx.gemm_int8(x.clone(memory_format=torch.contiguous_format) if K % 16 == 0 else x, sx, w, sw, bias, out_dtype=dtype)
        check(want, x, sx, w, sw, bias)
        for pad, shift in ((0, 1), (3, 0), (8, 0), (24, 8)):
            flat = torch.full((M * (N + pad) + shift,), 9.0, device="cuda", dtype=dtype)
            full = flat[shift:].view(M, N + pad)
            ctx.gemm_int8(x, sx, w, sw, bias, out=full[:, :N])
            assert torch.equal(full[:, :N], want)
            assert (full[:, N:] == 9).all() and (flat[:shift] == 9).all()
    assert ctx.status() == 0


def test_all_codes_and_the_longest_contraction(ctx):
    # -128 is a code too; 131071 * 128 * 128 is the largest sum that fits
    K = 131071
    x = torch.full((3, 131072), -128, dtype=torch.int8, device="cuda")[:, :K]
    w = torch.full((2, 131072), -128, dtype=torch.int8, device="cuda")[:, :K]
    w[1] = 127
    one3, one2 = torch.ones(3, device="cuda"), torch.ones(2, device="cuda")
    z = ctx.gemm_int8(x, one3, w, one2)
    assert z[0].tolist() == [float(torch.tensor(131071 * 16384).float()), float(torch.tensor(-131071 * 128 * 127).float())]
    assert torch.equal(z, z[:1].expand(3, 2))
    with pytest.raises(binding.LuqError) as e:
        ctx.gemm_int8(torch.zeros(1, 131072, dtype=torch.int8, device="cuda"), one3[:1], torch.zeros(1, 131072, dtype=torch.int8, device="cuda"), one2[:1])
    assert e.value.code == binding.ERR_UNSUPPORTED


def test_what_lies_behind_a_row_is_not_read(ctx):
    # codes beyond K, rows beyond M and N, and a row's pad hold anything
    M, N, K = 70, 200, 100
    x, w = codes(M, K, 5, ld=144), codes(N, K, 6, ld=144)
    sx, sw = floats(M, 1), floats(N, 2)
    want = ctx.gemm_int8(x, sx, w, sw)
    big_x, big_w = codes(M + 60, K, 7, ld=144), codes(N + 60, K, 8, ld=144)
    big_x[:M], big_w[:N] = x, w
    assert torch.equal(ctx.gemm_int8(big_x[:M], sx, big_w[:N], sw), want)


def test_empty(ctx):
    w, sw = codes(64, 32, 1), floats(64, 2)
    assert ctx.gemm_int8(codes(0, 32, 1), floats(0, 1), w, sw).shape == (0, 64)
    assert ctx.gemm_int8(codes(5, 32, 1), floats(5, 1), codes(0, 32, 1), floats(0, 1)).shape == (5, 0)
    assert ctx.quant_int8_gemm(torch.empty(0, 32, device="cuda"), w, sw).shape == (0, 64)
    launches = ctx.launches
    ctx.gemm_int8(codes(0, 32, 1), floats(0, 1), w, sw)
    assert ctx.launches == launches


def grouped_check(ctx, sizes, N, K, lead=0, tail=0, bias=True, w_gap=0, seed=0):
    E, M = len(sizes), lead + sum(sizes) + tail
    x = codes(M, K, seed + 1)
    w = codes(N + w_gap, K, seed + 2, lead=(E,))[:, :N]
    sx, sw = floats(M, seed + 3), floats(E * N, seed + 4).view(E, N)
    b = floats(E * N, seed + 5).view(E, N) - 0.01 if bias else None
    ends = [lead]
    for n in sizes:
        ends.append(ends[-1] + n)
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        z = torch.full((M, N), 5.0, device="cuda", dtype=dtype)
        ctx.gemm_int8_grouped(x, sx, offsets, w, sw, b, out=z)
        for e in range(E):
            i, j = ends[e], ends[e + 1]
            if j > i:
                check(z[i:j], x[i:j], sx[i:j], w[e], sw[e], None if b is None else b[e])
        assert (z[:lead] == 5).all() and (z[M - tail:] == 5).all()
    assert ctx.status() == 0


@pytest.mark.parametrize("sizes", [[1], [0, 1], [1, 0, 0, 2], [16, 17, 15, 0, 33], [128, 0, 127, 129, 1], [300, 1, 700], [0, 0, 0, 5],
                                   [513, 511], [64] * 9, [1] * 40, [0] * 31 + [3] + [0] * 40 + [70], [1000, 2, 2, 2, 2, 2, 2, 2],
                                   [257, 255, 256, 31, 32, 33, 2000]])
def test_grouped(ctx, sizes):
    grouped_check(ctx, sizes, 136, 80)
    grouped_check(ctx, sizes, 129, 100, lead=3, tail=5, bias=False, w_gap=2, seed=7)
    grouped_check(ctx, sizes, 520, 384, lead=1, seed=9)


def test_grouped_with_many_groups(ctx):
    g = torch.Generator().manual_seed(1)
    sizes = torch.randint(0, 4, (1024,), generator=g).tolist()
    grouped_check(ctx, sizes, 48, 32)
    sizes = [0] * 1024
    sizes[1000] = 37
    grouped_check(ctx, sizes, 48, 32)


def test_no_group_has_rows(ctx):
    w, sw = codes(64, 32, 1, lead=(3,)), floats(192, 2).view(3, 64)
    z = torch.full((7, 64), 5.0, device="cuda")
    ctx.gemm_int8_grouped(codes(7, 32, 1), floats(7, 1), torch.full((4,), 4, dtype=torch.int32, device="cuda"), w, sw, out=z)
    assert (z == 5).all() and ctx.status() == 0


def test_offsets_that_are_not_offsets(ctx):
    # decreasing or out of range: the running maximum, clamped to [0, M]; the status word says so
    M, N, K, E = 200, 96, 64, 5
    x, w = codes(M, K, 1), codes(N, K, 2, lead=(E,))
    sx, sw = floats(M, 3), floats(E * N, 4).view(E, N)
    for bad in ([-5, 20, 10, 60, 2 ** 31 - 1, 7], [0, 300, 400, 100, 50, 60], [-2 ** 31, -7, -6, -5, -4, -3], [200, 0, 0, 0, 0, 0]):
        fixed, top = [], 0
        for v in bad:
            top = max(top, min(max(v, 0), M))
            fixed.append(top)
        z, want = torch.full((M, N), 5.0, device="cuda"), torch.full((M, N), 5.0, device="cuda")
        ctx.gemm_int8_grouped(x, sx, torch.tensor(fixed, dtype=torch.int32, device="cuda"), w, sw, out=want)
        assert ctx.status() == 0
        ctx.gemm_int8_grouped(x, sx, torch.tensor(bad, dtype=torch.int32, device="cuda"), w, sw, out=z)
        assert ctx.status() == binding.STATUS_OFFSETS
        assert torch.equal(z, want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", [(1, 4096, 1024), (1, 300, 77), (4, 4096, 4096), (7, 128, 130), (40, 1000, 520), (333, 257, 1000),
                                   (1500, 640, 768)])
def test_one_call_equals_two(ctx, M, N, K, dtype):
    g = torch.Generator("cuda").manual_seed(M + N + K)
    x = torch.randn(M, K + 3, device="cuda", generator=g).to(dtype)
    w, sw = ctx.quant_int8_rows(torch.randn(N, K, device="cuda", generator=g))
    gamma, beta, bias = (torch.randn(n, device="cuda", generator=g) for n in (K, K, N))
    for xx in (x[:, :K], x[:, :K].contiguous(), x[:, 3:]):
        for out_dtype in (torch.float32, torch.bfloat16):
            q, s = ctx.quant_int8_rows(xx)
            assert torch.equal(ctx.quant_int8_gemm(xx, w, sw, bias, out_dtype=out_dtype), ctx.gemm_int8(q, s, w, sw, bias, out_dtype=out_dtype))
            q, s = ctx.layer_norm_int8(xx, gamma, beta, 1e-5)
            assert torch.equal(ctx.layer_norm_int8_gemm(xx, gamma, beta, 1e-5, w, sw, bias, out_dtype=out_dtype),
                               ctx.gemm_int8(q, s, w, sw, bias, out_dtype=out_dtype))
    assert ctx.quant_int8_gemm(x[:, :K], w, sw).dtype == dtype
    # and grouped: three experts, one of them without rows
    E = 3
    w3 = torch.stack([codes(N, K, e, ld=-(-K // 16) * 16 + 16).as_strided((N, -(-K // 16) * 16), (-(-K // 16) * 16 + 16, 1)) for e in range(E)])[:, :, :K]
    sw3 = floats(E * N, 3).view(E, N)
    offsets = torch.tensor([0, M // 2, M // 2, M], dtype=torch.int32, device="cuda")
    q, s = ctx.quant_int8_rows(x[:, :K])
    assert torch.equal(ctx.quant_int8_gemm_grouped(x[:, :K], offsets, w3, sw3), ctx.gemm_int8_grouped(q, s, offsets, w3, sw3, out_dtype=dtype))
    assert ctx.status() == 0


def test_a_token_with_nan_stays_alone(ctx):
    x = torch.randn(40, 256, device="cuda")
    w, sw = ctx.quant_int8_rows(torch.randn(192, 256, device="cuda"))
    want = ctx.quant_int8_gemm(x, w, sw)
    x[7, 3] = float("nan")
    x[20, 255] = float("inf")
    z = ctx.quant_int8_gemm(x, w, sw)
    assert ctx.status() == binding.STATUS_NONFINITE
    assert torch.isnan(z[7]).all() and torch.isnan(z[20]).all()
    keep = [i for i in range(40) if i not in (7, 20)]
    assert torch.equal(z[keep], want[keep])


def test_another_stream_and_a_graph(ctx):
    x = torch.randn(64, 512, device="cuda")
    w, sw = ctx.quant_int8_rows(torch.randn(256, 512, device="cuda"))
    want = ctx.quant_int8_gemm(x, w, sw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        z = ctx.quant_int8_gemm(x, w, sw)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(z, want)
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.quant_int8_gemm(x, w, sw, out=out)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and ctx.status() == 0


def test_sm_limit_changes_nothing(ctx):
    x, w = codes(700, 300, 1), codes(520, 300, 2)
    sx, sw = floats(700, 3), floats(520, 4)
    want = ctx.gemm_int8(x, sx, w, sw)
    try:
        for n in (1, 2, 3, 50):
            ctx.set_option(binding.OPT_SM_LIMIT, n)
            assert torch.equal(ctx.gemm_int8(x, sx, w, sw), want)
            assert torch.equal(ctx.gemm_int8(x[:5], sx[:5], w, sw), want[:5])
    finally:
        ctx.set_option(binding.OPT_SM_LIMIT, 0)
    assert ctx.status() == 0


def test_repeats_bit_for_bit(ctx):
    for M, N, K in ((3, 2048, 4096), (200, 512, 1024), (1000, 1024, 640)):
        x, w = codes(M, K, 1), codes(N, K, 2)
        sx, sw = floats(M, 3), floats(N, 4)
        want = ctx.gemm_int8(x, sx, w, sw)
        for _ in range(100):
            assert torch.equal(ctx.gemm_int8(x, sx, w, sw), want)
    assert ctx.status() == 0


def test_more_than_2_to_31_outputs(ctx):
    M, N, K = 70_000, 32_768, 16
    x, w = codes(M, K, 1), codes(N, K, 2)
    x[-300:] = x[:300]
    sx, sw = floats(M, 3), floats(N, 4)
    sx[-300:] = sx[:300]
    z = ctx.gemm_int8(x, sx, w, sw, out_dtype=torch.bfloat16)
    check(z[:300], x[:300], sx[:300], w, sw, None)
    assert torch.equal(z[-300:], z[:300])
    odd = torch.empty(M, N + 1, device="cuda", dtype=torch.bfloat16)[:, :N]         # rows TMA cannot address
    ctx.gemm_int8(x, sx, w, sw, out=odd)
    assert torch.equal(odd[-300:], z[:300]) and ctx.status() == 0


def test_refusals(ctx):
    x, w = codes(8, 64, 1), codes(32, 64, 2)
    sx, sw = floats(8, 1), floats(32, 2)
    bad_rows = torch.zeros(8, 72, dtype=torch.int8, device="cuda")[:, :64]
    for call in (lambda: ctx.gemm_int8(bad_rows, sx, w, sw), lambda: ctx.gemm_int8(x.float(), sx, w, sw),
                 lambda: ctx.gemm_int8(x, sx[:7], w, sw), lambda: ctx.gemm_int8(x, sx, w, sw.double()),
                 lambda: ctx.gemm_int8(x, sx, codes(32, 48, 1), sw), lambda: ctx.gemm_int8(x, sx, w, sw, bias=sw[:5]),
                 lambda: ctx.gemm_int8(x, sx, w, sw, out_dtype=torch.float16), lambda: ctx.gemm_int8(x, sx, w.cpu(), sw),
                 lambda: ctx.gemm_int8(x, sx, w, sw, out=torch.empty(32, 8, device="cuda").t()),
                 lambda: ctx.gemm_int8_grouped(x, sx, torch.zeros(2, dtype=torch.int64, device="cuda"), w[None], sw[None]),
                 lambda: ctx.gemm_int8_grouped(x, sx, torch.zeros(3, dtype=torch.int32, device="cuda"), w[None], sw[None]),
                 lambda: ctx.gemm_int8_grouped(x, sx, torch.zeros(2, dtype=torch.int32), w[None], sw[None]),
                 lambda: ctx.quant_int8_gemm(torch.zeros(8, 63, device="cuda"), w, sw),
                 lambda: ctx.quant_int8_gemm(torch.zeros(8, 64, device="cuda").half(), w, sw)):
        with pytest.raises(TypeError):
            call()
    many = torch.zeros(1025, 1, 16, dtype=torch.int8, device="cuda")
    with pytest.raises(binding.LuqError) as e:
        ctx.gemm_int8_grouped(codes(1, 16, 1), floats(1, 1), torch.zeros(1026, dtype=torch.int32, device="cuda"), many, floats(1025, 1).view(1025, 1))
    assert e.value.code == binding.ERR_ARG
    wide = torch.empty(1100, 100_000, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(binding.LuqError) as e:
        ctx.quant_int8_gemm(wide, torch.zeros(4, 100_000, dtype=torch.int8, device="cuda"), floats(4, 1))
    assert e.value.code == binding.ERR_WORKSPACE
    L, s = binding.load(), torch.cuda.current_stream().cuda_stream
    z = torch.empty(8, 32, device="cuda")
    good = dict(x=x.data_ptr(), ldx=64, sx=sx.data_ptr(), w=w.data_ptr(), ldw=64, sw=sw.data_ptr(), b=None, z=z.data_ptr(), zt=0, ldz=32, M=8, N=32, K=64)
    call = lambda k: L.luq_gemm_int8(ctx.handle, k["x"], k["ldx"], k["sx"], k["w"], k["ldw"], k["sw"], k["b"], k["z"], k["zt"], k["ldz"], k["M"], k["N"], k["K"], s)  # noqa: E731
    assert call(good) == 0
    for key, value in (("x", None), ("x", x.data_ptr() + 8), ("ldx", 72), ("ldx", 48), ("sx", None), ("w", None), ("ldw", 63), ("sw", None),
                       ("sw", sw.data_ptr() + 2), ("z", None), ("z", z.data_ptr() + 1), ("zt", 2), ("ldz", 31), ("M", -1), ("N", -1), ("K", 0), ("M", 1 << 31)):
        assert call(dict(good, **{key: value})) == binding.ERR_ARG, (key, value)
    assert ctx.status() == 0
