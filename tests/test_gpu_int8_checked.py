"""The bounds-checking build's checks in the row kernels and the int8 product: each kernel reports accesses to a row's last
element when rows are declared one element shorter than they are (nothing out of range is accessed: the element is
there, and the access is skipped), and nothing otherwise."""
import os
import subprocess
import sys

import pytest

from paper_2112_10769_b200 import binding
from paper_2112_10769_b200 import build as lib_build

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r'''
import torch
from paper_2112_10769_b200 import binding
assert binding.debug_build()
ctx = binding.Context(0)
g = torch.Generator("cuda").manual_seed(1)
r = lambda *s: torch.randn(*s, device="cuda", generator=g)

def fires(call, *what):
    ctx.set_option(binding.OPT_CHECK_SLACK, 1)
    call()
    assert ctx.status() & binding.STATUS_BOUNDS, what
    ctx.set_option(binding.OPT_CHECK_SLACK, 0)
    call()
    assert ctx.status() == 0, what

# rows by 16-byte loads, element by element, through the rings, whole, full and ragged; wider than registers hold
for rows, cols, pad, shift in ((3, 64, 0, 0), (3, 100, 0, 1), (40, 255, 2, 0), (3, 768, 0, 0), (3, 1024, 0, 0), (3, 1536, 0, 0), (2, 4096, 0, 0),
                               (5, 1025, 0, 0), (1300, 301, 0, 0), (1300, 704, 0, 0), (1300, 1024, 0, 0), (2000, 771, 5, 0), (1300, 4096, 0, 0),
                               (1300, 1025, 0, 1), (2, 9000, 0, 0), (700, 16384, 0, 0), (3, 20000, 0, 0), (700, 20001, 0, 1)):
    for dtype in (torch.float32, torch.bfloat16):
        x, dy = (r(rows * (cols + pad) + shift).to(dtype)[shift:].view(rows, cols + pad)[:, :cols] for _ in range(2))
        w, b = r(cols), r(cols)
        _, mean, rstd = ctx.layer_norm(x, w, b)
        for call in (lambda: ctx.layer_norm(x, w, b), lambda: ctx.layer_norm(x), lambda: ctx.layer_norm_int8(x, w, b), lambda: ctx.quant_int8_rows(x),
                     lambda: ctx.layer_norm_bwd(dy, x, mean, rstd, w),
                     lambda: ctx.layer_norm_bwd(dy, x, mean, rstd, w, need_dweight=False, need_dbias=False)):
            fires(call, rows, cols, pad, shift, dtype)
# products of every tile: 16 to 256 tokens, split and not, copies and single stores
for M, N, K in ((1, 4096, 1024), (8, 130, 64), (300, 8200, 64), (20, 130, 1000), (70, 257, 640), (333, 500, 1300), (2000, 640, 128), (4000, 4096, 256)):
    w, sw = ctx.quant_int8_rows(r(2 * N, K))
    q, s = ctx.quant_int8_rows(r(M, K))
    w2 = w.as_strided((2, N, K), (N * w.stride(0), w.stride(0), 1))
    offsets = torch.tensor([0, M // 3, M], dtype=torch.int32, device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        fires(lambda: ctx.gemm_int8(q, s, w[:N], sw[:N], out_dtype=dtype), M, N, K)
        fires(lambda: ctx.gemm_int8_grouped(q, s, offsets, w2, sw.view(2, N), out_dtype=dtype), M, N, K)
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


def test_the_normal_build_has_no_such_option():
    ctx = binding.Context(0)
    with pytest.raises(binding.LuqError) as e:
        ctx.set_option(binding.OPT_CHECK_SLACK, 1)
    assert e.value.code == binding.ERR_UNSUPPORTED
    ctx.close()
