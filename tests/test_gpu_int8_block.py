"""The 8-bit modules, the layer norm module, and the example that trains a block in 4 bits and answers in 8."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2112_10769_b200 import autograd, binding
from paper_2112_10769_b200 import build as lib_build

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_layer_norm_module_trains_like_its_formula():
    # 3-D input, parameters in 32 bits; the gradients of the formula in 64 bits.  u = 2^-24; sums over 2 x 33 rows
    # and 96 columns: 200 u covers every chain of roundings, relative to the largest entries
    g = torch.Generator("cuda").manual_seed(3)
    x = torch.randn(2, 33, 96, device="cuda", generator=g, requires_grad=True)
    m = autograd.LayerNorm(96, device="cuda")
    with torch.no_grad():
        m.weight.copy_(torch.rand(96, device="cuda", generator=g) + 0.5)
        m.bias.copy_(torch.rand(96, device="cuda", generator=g))
    dy = torch.randn(2, 33, 96, device="cuda", generator=g)
    m(x).backward(dy)
    x64, w64, b64 = (t.detach().double().requires_grad_() for t in (x, m.weight, m.bias))
    y64 = (x64 - x64.mean(-1, keepdim=True)) * (x64.var(-1, unbiased=False, keepdim=True) + m.eps).rsqrt() * w64 + b64
    y64.backward(dy.double())
    for got, ref in ((m(x), y64), (x.grad, x64.grad), (m.weight.grad, w64.grad), (m.bias.grad, b64.grad)):
        assert (got.double() - ref).abs().max() <= 200 * 2 ** -24 * ref.abs().max()
    # a broadcast gradient, and no gradient for what does not need one
    m.weight.requires_grad_(False)
    m.weight.grad = None
    x.grad = None
    m(x).sum().backward()
    assert m.weight.grad is None and x.grad is not None
    assert autograd.LayerNorm(96, bias=False, device="cuda")(x.bfloat16()).dtype == torch.bfloat16


def test_int8_linear_and_experts():
    from paper_2112_10769_b200.int8 import Int8Experts, Int8Linear
    g = torch.Generator("cuda").manual_seed(5)
    lin = torch.nn.Linear(200, 72, device="cuda")
    norm = torch.nn.LayerNorm(200, device="cuda")
    x = torch.randn(3, 7, 200, device="cuda", generator=g)
    with torch.no_grad():
        # a token's and a channel's largest error is half a step of 127 each: relative to |x| |w| below 1 / 127
        for layer, want in ((Int8Linear.of(lin), lin(x)), (Int8Linear.of(lin, norm=norm), lin(norm(x)))):
            z = layer(x)
            assert z.shape == want.shape and (z - want).norm() <= want.norm() / 60
        w = torch.randn(4, 72, 200, device="cuda", generator=g)
        layer = Int8Experts(w)
        expert = torch.tensor([3, 0, 3, 1, 1, 0, 3], device="cuda")
        rows = x.reshape(-1, 200)[:7]
        z = layer.route(rows, expert)
        want = torch.einsum("tk,tnk->tn", rows, w[expert])
        assert (z - want).norm() <= want.norm() / 60
        # an expert's rows as the dense layer computes them
        for e in (0, 1, 3):
            at = (expert == e).nonzero()[:, 0]
            assert torch.equal(z[at], Int8Linear(w[e])(rows[at]))
    with pytest.raises(ValueError):
        Int8Linear.of(lin, norm=torch.nn.LayerNorm(199, device="cuda"))


def test_codes_and_scales_of_a_call_are_its_own():
    # the token codes and scales of a call live in the context's workspace: calls that follow one another without a
    # pause, each with other inputs, must not see one another's
    ctx = binding.Context(0)
    for M, N, K in ((1, 4096, 1024), (4, 1024, 4096), (40, 512, 512), (300, 1024, 256)):
        g = torch.Generator("cuda").manual_seed(M)
        w, sw = ctx.quant_int8_rows(torch.randn(N, K, device="cuda", generator=g))
        gamma = torch.rand(K, device="cuda", generator=g) + 0.5
        xs = [torch.randn(M, K, device="cuda", generator=g) * 10.0 ** i for i in range(-2, 3)]
        want = []
        for x in xs:
            for q, s in (ctx.quant_int8_rows(x), ctx.layer_norm_int8(x, gamma)):
                want.append(ctx.gemm_int8(q, s, w, sw))
                torch.cuda.synchronize()
        for _ in range(40):
            got = []
            for x in xs:
                got.append(ctx.quant_int8_gemm(x, w, sw))
                got.append(ctx.layer_norm_int8_gemm(x, gamma, None, 1e-5, w, sw))
            assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert ctx.status() == 0
    ctx.close()


def test_example():
    from paper_2112_10769_b200 import example_block
    r = example_block.main(width=128, tokens=512, steps=40, verbose=False)
    assert r["status"] == 0 and r["one_token_equals_prompt"]
    assert r["last_loss"] < 0.8 * r["first_loss"]
    assert r["int8_error"] < 0.05 and r["expert_error"] < 0.05


CHILD = r'''
import torch
from paper_2112_10769_b200 import binding
assert binding.debug_build()
ctx = binding.Context(0)
g = torch.Generator("cuda").manual_seed(1)
r = lambda *s: torch.randn(*s, device="cuda", generator=g)
for rows, cols in ((3, 7), (40, 255), (1300, 520), (5, 1024), (2000, 771), (2, 9000)):
    for dtype in (torch.float32, torch.bfloat16):
        x, w = r(rows, cols + 3).to(dtype)[:, :cols], r(cols)
        y, mean, rstd = ctx.layer_norm(x, w, w)
        ctx.layer_norm_bwd(y, x, mean, rstd, w)
        ctx.layer_norm_int8(x, w, w)
        ctx.quant_int8_rows(x)
        assert ctx.status() == 0, (rows, cols)
for M, N, K in ((1, 300, 100), (17, 129, 1000), (70, 257, 640), (333, 500, 130), (1100, 1000, 300)):
    w, sw = ctx.quant_int8_rows(r(N, K))
    w3, sw3 = ctx.quant_int8_rows(r(3 * N, K))
    w3 = w3.as_strided((3, N, K), (N * w3.stride(0), w3.stride(0), 1))
    offsets = torch.tensor([0, M // 3, M // 3, M], dtype=torch.int32, device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        x = r(M, K).to(dtype)
        z = ctx.quant_int8_gemm(x, w, sw)
        q, s = ctx.quant_int8_rows(x)
        ref = (q.double() @ w.double().t()) * s.double()[:, None] * sw.double()
        assert (z.double() - ref).abs().max() <= 2.0 ** -7 * ref.abs().max()
        ctx.quant_int8_gemm_grouped(x, offsets, w3, sw3.view(3, N))
        assert ctx.status() == 0, (M, N, K)
print("checked build ok")
'''


def test_bounds_checking_build_finds_nothing():
    lib = lib_build.LIB_DEBUG
    if not os.path.exists(lib):
        lib = lib_build.build(debug=True)
    env = dict(os.environ, LUQ_LIB=lib, PYTHONPATH=ROOT + os.pathsep + os.environ.get("PYTHONPATH", ""))
    out = subprocess.run([sys.executable, "-c", CHILD], env=env, cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert out.returncode == 0, out.stdout[-2000:] + out.stderr[-4000:]
    assert "checked build ok" in out.stdout
