"""The bounds-checking build's checks in the e2m1 and expert kernels: each reports accesses to the last elements of rows that are declared
shorter than they are (nothing out of range is accessed: the elements are there, and the access is skipped), and nothing otherwise."""
import os
import subprocess
import sys

import pytest

from paper_2112_10769_b200 import build as lib_build

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r'''
import torch
from paper_2112_10769_b200 import binding, e2m1
assert binding.debug_build()
ctx = binding.Context(0)
g = torch.Generator("cuda").manual_seed(1)
r = lambda *s: torch.randn(*s, device="cuda", generator=g)

def fires(call, *what):
    ctx.set_option(binding.OPT_CHECK_SLACK, 2)
    call()
    assert ctx.status() & binding.STATUS_BOUNDS, what
    ctx.set_option(binding.OPT_CHECK_SLACK, 0)
    call()
    assert ctx.status() == 0, what

for rows, cols, pad, shift in ((3, 64, 0, 0), (700, 100, 0, 1), (40, 255, 2, 0), (3, 1024, 0, 0), (700, 1000, 0, 0), (2, 4097, 0, 0), (700, 4096, 0, 0), (2, 33001, 0, 1)):
    for dtype in (torch.float32, torch.bfloat16):
        x = r(rows * (cols + pad) + shift).to(dtype)[shift:].view(rows, cols + pad)[:, :cols]
        for block in (16, 32):
            fires(lambda: ctx.quant_e2m1_rows(x, block), rows, cols, dtype, block)
for M, N, K in ((1, 4096, 1024), (2, 130, 64), (8, 130, 64), (300, 8200, 64), (70, 257, 640), (333, 500, 1300), (2000, 640, 128), (4000, 4096, 256)):
    x, w = r(M, K), r(2, N, K)
    offsets = torch.tensor([0, M // 3, M], dtype=torch.int32, device="cuda")
    for block in (16, 32):
        wq, we = e2m1.quantize_weight(w[0], block), e2m1.quantize_weight(w, block)
        q, qe = ctx.quant_e2m1_rows(x, block), ctx.quant_e2m1_rows(x, block, offsets=offsets)
        for dtype in (torch.float32, torch.bfloat16):
            fires(lambda: ctx.gemm_e2m1(*q, *wq, block=block, out_dtype=dtype), M, N, K)
            fires(lambda: ctx.quant_e2m1_gemm(x, *wq, block=block, out_dtype=dtype), M, N, K)
            fires(lambda: ctx.gemm_e2m1_grouped(*qe, offsets, *we, block=block, out_dtype=dtype), M, N, K)
for T, E, k in ((1, 256, 8), (50, 60, 4), (33, 1000, 9), (70, 8, 2), (40, 100, 3)):
    for dtype in (torch.float32, torch.bfloat16):
        x = r(T, E).to(dtype)
        chosen, w = ctx.route(x, k)
        fires(lambda: ctx.route(x, k), T, E)
        fires(lambda: ctx.route_bwd(w, x, chosen, renormalize=False), T, E)
        fires(lambda: ctx.expert_order(chosen, E), T, E)
for T, cols, k in ((1, 64, 2), (50, 771, 3), (30, 1000, 2), (7, 4100, 1)):
    for dtype in (torch.float32, torch.bfloat16):
        x, y, w = r(T, cols).to(dtype), r(T * k, cols).to(dtype), r(T, k)
        offsets, position = ctx.expert_order(torch.rand(T, 8, device="cuda").topk(k, 1).indices.to(torch.int32), 8)
        fires(lambda: ctx.dispatch(x, position, offsets), T, cols)
        fires(lambda: ctx.combine(y, position, w, x), T, cols)
        fires(lambda: ctx.combine_bwd(x, y, position, w, offsets), T, cols)
ctx.close()
print("checks fire")
'''


def test_every_kernel_checks_its_rows():
    lib = lib_build.LIB_DEBUG
    if not os.path.exists(lib):
        lib = lib_build.build(debug=True)
    env = dict(os.environ, LUQ_LIB=lib, PYTHONPATH=ROOT + os.pathsep + os.environ.get("PYTHONPATH", ""))
    out = subprocess.run([sys.executable, "-c", CHILD], env=env, cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert out.returncode == 0, out.stdout[-2000:] + out.stderr[-4000:]
    assert "checks fire" in out.stdout
