"""The one-call 8-bit products as programs use them: more tokens than the workspace holds, several streams, graphs."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2112_10769_b200 import autograd, binding

pytestmark = pytest.mark.gpu
WORKSPACE = 96 << 20
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


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


def test_streams_answer_side_by_side():
    # two streams through the modules of one device, nothing waits for anything: neither sees the other's codes,
    # scales or partial sums.  The first calls' results, made one at a time, are the reference
    from paper_2112_10769_b200.int8 import Int8Experts, Int8Linear
    g = torch.Generator("cuda").manual_seed(1)
    K, N, E = 1024, 512, 4
    w = torch.randn(E, N, K, device="cuda", generator=g)
    dense, normed, experts = Int8Linear(w[0]), Int8Linear(w[1], norm=torch.nn.LayerNorm(K, device="cuda")), Int8Experts(w)
    gamma = torch.rand(K, device="cuda", generator=g) + 0.5
    lib = autograd.context(w.device)

    def calls(x, offsets):
        _, mean, rstd = lib.layer_norm(x, gamma)
        return (dense(x), normed(x), experts(x, offsets), *lib.layer_norm_bwd(x.flip(0), x, mean, rstd, gamma))

    streams = [torch.cuda.Stream() for _ in range(2)]
    inputs, want = [], []
    for i, rows in enumerate((700, 3000)):
        x = torch.randn(rows, K, device="cuda", generator=g) * 10.0 ** (2 * i)
        offsets = torch.tensor([0, rows // 5, rows // 2, rows // 2, rows], dtype=torch.int32, device="cuda")
        inputs.append((x, offsets))
        want.append(calls(x, offsets))
        torch.cuda.synchronize()
    got = [[], []]
    for _ in range(40):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(calls(*inputs[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for result in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(result, want[i]))
    assert lib.status() == 0


def test_a_graph_has_a_workspace_of_its_own(ctx):
    # a captured call is replayed while the stream it was captured from goes on with other tokens
    x, other = (torch.randn(2000, 1024, device="cuda") * f for f in (1, 100))
    w, sw = ctx.quant_int8_rows(torch.randn(256, 1024, device="cuda"))
    want, want_other = ctx.quant_int8_gemm(x, w, sw), ctx.quant_int8_gemm(other, w, sw)
    out = torch.empty_like(want)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        for _ in range(20):
            ctx.quant_int8_gemm(x, w, sw, out=out)
    replay = torch.cuda.Stream()
    for _ in range(10):
        with torch.cuda.stream(replay):
            out.zero_()
            graph.replay()
        with torch.cuda.stream(stream):
            got = [ctx.quant_int8_gemm(other, w, sw) for _ in range(20)]
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all(torch.equal(z, want_other) for z in got)
    assert ctx.status() == 0


NO_MEMORY = r"""
import torch
from paper_2112_10769_b200 import binding
ctx = binding.Context(0)
M, N, K = 12000, 64, 8192
x = torch.randn(M, K, device="cuda")
w, sw = ctx.quant_int8_rows(torch.randn(N, K, device="cuda"))
want, out = ctx.quant_int8_gemm(x, w, sw), torch.zeros(M, N, device="cuda")
torch.cuda.synchronize()
torch.cuda.empty_cache()
torch.cuda.set_per_process_memory_fraction(1e-6)
launches = ctx.launches
try:
    ctx.quant_int8_gemm(x, w, sw, out=out)
except torch.OutOfMemoryError:
    print("no memory")
assert ctx.launches == launches
torch.cuda.set_per_process_memory_fraction(1.0)
ctx.quant_int8_gemm(x, w, sw, out=out)
assert torch.equal(out, want) and ctx.status() == 0
"""


def test_no_memory_for_a_workspace_is_torchs_error():
    # (a limit of torch's allocator, not of the device: nothing is filled up.  A process of its own: what other tests
    # left in the allocator would do for a workspace)
    out = subprocess.run([sys.executable, "-c", NO_MEMORY], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and "no memory" in out.stdout, out.stdout[-2000:] + out.stderr[-4000:]


def test_modules_answer_the_same_after_a_move_and_a_cast():
    import copy
    from paper_2112_10769_b200.int8 import Int8Experts, Int8Linear
    K = 200                                               # rows of codes with eight bytes between them
    x, offsets = torch.randn(9, K, device="cuda"), torch.tensor([0, 4, 9], dtype=torch.int32, device="cuda")
    dense = Int8Linear(torch.randn(72, K, device="cuda"), torch.randn(72, device="cuda"), torch.nn.LayerNorm(K, device="cuda"))
    experts = Int8Experts(torch.randn(2, 72, K, device="cuda"))
    norm = autograd.LayerNorm(K, device="cuda")
    want = dense(x), experts(x, offsets), norm(x)
    for moved in (lambda m: m.cpu().cuda(), lambda m: m.bfloat16(), lambda m: m.half(), copy.deepcopy):
        got = moved(dense)(x), moved(experts)(x, offsets), moved(norm)(x)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert norm(x.bfloat16()).dtype == torch.bfloat16


def test_the_stride_between_groups_means_nothing_for_one_group(ctx):
    M, N, K = 20, 48, 64
    x, w = (torch.randint(-127, 128, (n, K), device="cuda", dtype=torch.int8) for n in (M, N))
    sx, sw = torch.rand(M, device="cuda"), torch.rand(N, device="cuda")
    offsets = torch.tensor([0, M], dtype=torch.int32, device="cuda")
    want = ctx.gemm_int8(x, sx, w, sw)
    for stride in (N * K, 0, -16, 16):
        z = torch.zeros(M, N, device="cuda")
        rc = binding.load().luq_gemm_int8_grouped(ctx.handle, x.data_ptr(), K, sx.data_ptr(), offsets.data_ptr(), 1, w.data_ptr(), K, stride,
                                                  sw.data_ptr(), None, z.data_ptr(), 0, N, M, N, K, torch.cuda.current_stream().cuda_stream)
        assert rc == 0 and torch.equal(z, want), stride
    assert ctx.status() == 0
