"""The one-call 8-bit products as programs use them: more tokens than the workspace holds."""
import pytest
import torch

from paper_2112_10769_b200 import autograd, binding

pytestmark = pytest.mark.gpu
WORKSPACE = 96 << 20


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def tokens(rows, cols, dtype, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn(rows, cols, device="cuda", generator=g) * (1 + torch.rand(rows, 1, device="cuda", generator=g))).to(dtype)


# one call is the two calls bit for bit, whatever the number of rows: codes of 97 to 197 MiB, odd sizes among them
@pytest.mark.parametrize("M,N,K,dtype", [(14219, 384, 7232, torch.float32), (16384, 130, 8192, torch.bfloat16), (7101, 65, 14336, torch.bfloat16),
                                         (65536, 8, 1613, torch.bfloat16), (2100, 16, 98288, torch.bfloat16)])
def test_more_codes_than_the_workspace_holds(ctx, M, N, K, dtype):
    assert M * (-(-K // 16) * 16 + 4) > WORKSPACE
    x = tokens(M, K, dtype, M)
    w, sw = ctx.quant_int8_rows(torch.randn(N, K, device="cuda"))
    gamma, beta, bias = (torch.randn(n, device="cuda") for n in (K, K, N))
    q, s = ctx.quant_int8_rows(x)
    assert torch.equal(ctx.quant_int8_gemm(x, w, sw, bias), ctx.gemm_int8(q, s, w, sw, bias, out_dtype=dtype))
    q, s = ctx.layer_norm_int8(x, gamma, beta, 1e-5)
    wide = torch.full((M, N + 3), 5.0, device="cuda")
    ctx.layer_norm_int8_gemm(x, gamma, beta, 1e-5, w, sw, bias, out=wide[:, :N])
    assert torch.equal(wide[:, :N], ctx.gemm_int8(q, s, w, sw, bias)) and (wide[:, N:] == 5).all()
    assert ctx.status() == 0


@pytest.mark.parametrize("ends", [[0, 9000, 9000, 9001, 16384], [5, 7, 8191, 8193, 16000], [0, 0, 0, 0, 16384], [16384] * 5, [0, 20000, 5, 12000, 16384]])
def test_more_codes_than_the_workspace_holds_grouped(ctx, ends):
    # groups that begin, end, and are cut where a chunk of the rows ends; rows of no group; offsets that are none
    M, N, K, E = 16384, 72, 6200, 4
    assert M * (-(-K // 16) * 16 + 4) > WORKSPACE
    x = tokens(M, K, torch.bfloat16, 3)
    w, sw = ctx.quant_int8_rows(torch.randn(E * N, K, device="cuda"))
    w = w.as_strided((E, N, K), (N * w.stride(0), w.stride(0), 1))
    sw, bias = sw.view(E, N), torch.randn(E, N, device="cuda")
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    q, s = ctx.quant_int8_rows(x)
    got, want = (torch.full((M, N), 5.0, device="cuda") for _ in range(2))
    ctx.gemm_int8_grouped(q, s, offsets, w, sw, bias, out=want)
    flags = ctx.status()
    assert flags == (binding.STATUS_OFFSETS if ends[1] > M else 0)
    ctx.quant_int8_gemm_grouped(x, offsets, w, sw, bias, out=got)
    assert torch.equal(got, want) and ctx.status() == flags


def test_modules_answer_a_long_prompt():
    from paper_2112_10769_b200.int8 import Int8Experts, Int8Linear
    M, N, K = 8192, 40, 14336
    x, w = tokens(M, K, torch.bfloat16, 7), torch.randn(2, N, K, device="cuda")
    z = Int8Linear(w[0], norm=torch.nn.LayerNorm(K, device="cuda"))(x)
    for rows in (slice(0, 1), slice(4000, 4100), slice(M - 1, M)):
        assert torch.equal(z[rows], Int8Linear(w[0], norm=torch.nn.LayerNorm(K, device="cuda"))(x[rows]))
    z = Int8Experts(w)(x, torch.tensor([0, 5000, M], dtype=torch.int32, device="cuda"))
    assert torch.equal(z[:5000], Int8Linear(w[0])(x[:5000])) and torch.equal(z[5000:], Int8Linear(w[1])(x[5000:]))
    assert autograd.context(x.device).status() == 0
