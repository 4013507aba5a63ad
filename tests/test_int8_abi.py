"""Layer norm and 8-bit operators: what can be checked without a GPU."""
import ctypes

import pytest
import torch

from paper_2112_10769_b200 import binding
from paper_2112_10769_b200 import build as libbuild


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return binding.load()


def test_null_contexts_are_refused(lib):
    assert lib.luq_layer_norm(None, None, 0, 1, 1, 1, None, None, 0.0, None, 1, None, None, None) == binding.ERR_ARG
    assert lib.luq_layer_norm_bwd(None, None, 1, None, 1, 0, 1, 1, None, None, None, None, 1, None, None, None) == binding.ERR_ARG
    assert lib.luq_layer_norm_int8(None, None, 0, 1, 1, 1, None, None, 0.0, None, 16, None, None) == binding.ERR_ARG
    assert lib.luq_quant_int8_rows(None, None, 0, 1, 1, 1, None, 16, None, None) == binding.ERR_ARG
    product = [None, 0, 1, 1, 1, 16, None]
    assert lib.luq_gemm_int8(None, None, 16, None, None, 16, None, None, *product) == binding.ERR_ARG
    assert lib.luq_gemm_int8_grouped(None, None, 16, None, None, 1, None, 16, 16, None, None, *product) == binding.ERR_ARG
    assert lib.luq_quant_int8_gemm(None, None, 0, 16, None, 16, None, None, *product) == binding.ERR_ARG
    assert lib.luq_layer_norm_int8_gemm(None, None, 0, 16, None, None, 0.0, None, 16, None, None, *product) == binding.ERR_ARG
    assert lib.luq_quant_int8_gemm_grouped(None, None, 0, 16, None, 1, None, 16, 16, None, None, *product) == binding.ERR_ARG


def test_native_argument_handling_is_bound_to_the_library(lib):
    module = binding.native()
    x = torch.zeros(2, 16)
    ctx = ctypes.c_void_p(64).value        # never dereferenced: the tensors are refused first
    for call in (lambda: module.layer_norm(ctx, 0, x, None, None, 1e-5, None),
                 lambda: module.layer_norm_bwd(ctx, 0, x, x, x, x, None, True, True, True),
                 lambda: module.layer_norm_int8(ctx, 0, x, None, None, 1e-5),
                 lambda: module.quant_int8_rows(ctx, 0, x),
                 lambda: module.gemm_int8(ctx, 0, x, x, x, x, None, None, 0),
                 lambda: module.gemm_int8_grouped(ctx, 0, x, x, x, x, x, None, None, 0),
                 lambda: module.quant_int8_gemm(ctx, 0, x, x, x, None, None, -1),
                 lambda: module.layer_norm_int8_gemm(ctx, 0, x, None, None, 1e-5, x, x, None, None, -1),
                 lambda: module.quant_int8_gemm_grouped(ctx, 0, x, x, x, x, None, None, -1),
                 lambda: module.quant_int8_rows(ctx, 0, "x"), lambda: module.quant_int8_rows(ctx, 0),
                 lambda: module.quant_int8_rows("ctx", 0, x), lambda: module.quant_int8_rows(ctx, 0, None)):
        with pytest.raises(TypeError):
            call()
