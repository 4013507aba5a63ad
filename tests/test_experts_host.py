"""Microscaled 4-bit products and expert routing: what can be checked without a GPU."""
import ctypes

import pytest
import torch

from paper_2112_10769_b200 import binding, e2m1
from paper_2112_10769_b200 import build as libbuild


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return binding.load()


def test_null_contexts_are_refused(lib):
    product = [None, 0, 1, 1, 1, 64, None]                             # z, dtype, ld, M, N, K, stream
    weights, grouped = [None, 32, None, None, None], [None, 1, None, 32, 32, None, None, None]
    assert lib.luq_quant_e2m1_rows(None, None, 0, 1, 64, 64, 16, 1, None, 0, None, 1, None, 32, None, None, None) == binding.ERR_ARG
    assert lib.luq_gemm_e2m1(None, None, 32, None, None, 16, *weights, *product) == binding.ERR_ARG
    assert lib.luq_gemm_e2m1_grouped(None, None, 32, None, None, 16, *grouped, *product) == binding.ERR_ARG
    assert lib.luq_quant_e2m1_gemm(None, None, 0, 64, 16, *weights, *product) == binding.ERR_ARG
    assert lib.luq_quant_e2m1_gemm_grouped(None, None, 0, 64, 16, None, 1, *grouped, *product) == binding.ERR_ARG
    assert lib.luq_route(None, None, 0, 1, 8, 8, 2, 0, None, 1, 1, 2, 1, 1.0, None, None, None) == binding.ERR_ARG
    assert lib.luq_route_bwd(None, None, None, 0, 1, 8, 8, None, 2, 0, 1, 1.0, None, 8, None) == binding.ERR_ARG
    assert lib.luq_expert_order(None, None, 1, 2, 8, None, None, None) == binding.ERR_ARG
    assert lib.luq_dispatch(None, None, 0, 1, 8, 8, None, 2, None, 8, None, 8, None) == binding.ERR_ARG
    assert lib.luq_combine(None, None, 0, 2, 8, 8, None, 1, 2, None, None, 0, None, 8, None) == binding.ERR_ARG
    assert lib.luq_combine_bwd(None, None, 8, None, 8, 0, 2, 8, None, 1, 2, None, None, 8, None, 8, None, None) == binding.ERR_ARG


def test_native_argument_handling_refuses_host_tensors(lib):
    module = binding.native()
    x, i = torch.zeros(2, 16), torch.zeros(2, 2, dtype=torch.int32)
    ctx = ctypes.c_void_p(64).value                                    # never dereferenced: the tensors are refused first
    for call in (lambda: module.quant_e2m1_rows(ctx, 0, x, 16, 1, None, None), lambda: module.quant_e2m1_rows(ctx, 0, x),
                 lambda: module.gemm_e2m1(ctx, 0, x, x, x, x, x, x, None, 16, None, 0),
                 lambda: module.gemm_e2m1_grouped(ctx, 0, x, x, x, i, x, x, x, None, 16, None, 0),
                 lambda: module.quant_e2m1_gemm(ctx, 0, x, 16, x, x, x, None, None, -1),
                 lambda: module.quant_e2m1_gemm_grouped(ctx, 0, x, 16, i, i, x, x, x, None, None, -1),
                 lambda: module.route(ctx, 0, x, 2, 0, None, 1, 1, 2, True, 1.0),
                 lambda: module.route_bwd(ctx, 0, x, x, i, 0, True, 1.0),
                 lambda: module.expert_order(ctx, 0, i, 4), lambda: module.dispatch(ctx, 0, x, i, i, None),
                 lambda: module.combine(ctx, 0, x, i, None, None, None),
                 lambda: module.combine_bwd(ctx, 0, x, x, i, None, i, True, True),
                 lambda: module.route("ctx", 0, x, 2, 0, None, 1, 1, 2, True, 1.0), lambda: module.combine(ctx, 0, None, i, None, None, None)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(TypeError):
        binding._score("relu")


@pytest.mark.parametrize("rows,cols,block", [(1, 16, 16), (1, 1, 32), (127, 64, 16), (128, 129, 16), (129, 1000, 32), (333, 1000, 16), (260, 4096, 32)])
def test_scale_tiles(rows, cols, block):
    s = torch.randint(0, 255, (rows, -(-cols // block)), dtype=torch.uint8, generator=torch.Generator().manual_seed(rows))
    t = e2m1.scale_tiles(s, block)
    assert t.shape == (-(-rows // 128), -(-cols // (4 * block)), 512)
    assert torch.equal(e2m1.scale_rows(t, rows, cols, block), s)
    # the place of every scale, and zeros everywhere else
    for r in {0, rows // 2, rows - 1}:
        for b in {0, s.shape[1] // 2, s.shape[1] - 1}:
            assert t[r // 128, b // 4, 16 * (r % 32) + 4 * (r % 128 // 32) + b % 4] == s[r, b]
    assert t.sum(dtype=torch.int64) == s.sum(dtype=torch.int64)


def test_scale_tiles_of_several_matrices_follow_one_another():
    s = torch.randint(0, 255, (3, 130, 9), dtype=torch.uint8, generator=torch.Generator().manual_seed(1))
    t = e2m1.scale_tiles(s, 16)
    assert torch.equal(t, torch.cat([e2m1.scale_tiles(m, 16) for m in s]))
    assert torch.equal(e2m1.scale_tiles(s.view(torch.float8_e4m3fn), 16), t)


@pytest.mark.parametrize("block", [0, 8, 64])
def test_other_blocks_are_refused(block):
    with pytest.raises(ValueError):
        e2m1.scale_tiles(torch.zeros(1, 1, dtype=torch.uint8), block)
    with pytest.raises(ValueError):
        e2m1.quantize_weight(torch.zeros(16, 16), block)


def test_values_of_packed_numbers():
    # every code once, both halves of a byte, against the definition of e2m1
    codes = torch.arange(256, dtype=torch.uint8)[None, :]
    want = []
    for byte in range(256):
        for q in (byte & 15, byte >> 4):
            e, m = (q & 7) >> 1, q & 1
            v = 0.5 * m if e == 0 else (1 + 0.5 * m) * 2.0 ** (e - 1)
            want.append(-v if q & 8 else v)
    want = torch.tensor(want, dtype=torch.float64)[None, :]
    scales = torch.full((1, 16), 127 + 3, dtype=torch.uint8)
    assert torch.equal(e2m1.values(codes, e2m1.scale_tiles(scales, 32), None, 512, 32), 8 * want)
    scales = torch.full((1, 32), 1.5).to(torch.float8_e4m3fn)
    assert torch.equal(e2m1.values(codes, e2m1.scale_tiles(scales, 16), torch.tensor([0.25]), 512, 16), 0.375 * want)
