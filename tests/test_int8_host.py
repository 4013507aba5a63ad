"""The host side of layer norm and the 8-bit operators: contexts, modules and their buffers.  No GPU needed."""
import ctypes

import pytest
import torch

from paper_2112_10769_b200 import binding
from paper_2112_10769_b200 import build as libbuild


@pytest.fixture(scope="module", autouse=True)
def lib():
    libbuild.build()
    return binding.load()


def test_a_closed_context_is_refused(monkeypatch):
    # what a closed context owned has been freed: its address must not reach the library any more
    destroyed = []

    class Library:
        @staticmethod
        def luq_destroy(handle):
            destroyed.append(handle.value)

    ctx = binding.Context.__new__(binding.Context)
    ctx.device, ctx.handle, ctx._address, ctx._native = 0, ctypes.c_void_p(4096), 4096, binding.native()
    with monkeypatch.context() as m:
        m.setattr(binding, "load", lambda: Library)
        ctx.close()
    assert destroyed == [4096]
    x = torch.zeros(2, 16)
    for call in (lambda: ctx.layer_norm(x), lambda: ctx.layer_norm_bwd(x, x, x, x), lambda: ctx.layer_norm_int8(x),
                 lambda: ctx.quant_int8_rows(x), lambda: ctx.gemm_int8(x, x, x, x), lambda: ctx.gemm_int8_grouped(x, x, x, x, x),
                 lambda: ctx.quant_int8_gemm(x, x, x), lambda: ctx.layer_norm_int8_gemm(x, None, None, 1e-5, x, x),
                 lambda: ctx.quant_int8_gemm_grouped(x, x, x, x)):
        with pytest.raises(binding.LuqError) as e:
            call()
        assert e.value.code == binding.ERR_ARG


def test_a_context_takes_its_workspaces_from_torch(lib):
    # what lets calls on several streams share a context (the native half of Context.__init__)
    assert lib.luq_set_allocator(None, None, None, None) == binding.ERR_ARG
    with pytest.raises(binding.LuqError):
        binding.native().attach(0)


def test_a_second_derivative_of_layer_norm_is_refused(monkeypatch):
    # the backward pass is a kernel call that records nothing: differentiating through it has to raise, not to leave
    # the norm's part out.  The library's calls are played by the formulas here
    from paper_2112_10769_b200 import autograd

    class Formulas:
        @staticmethod
        def layer_norm(x, weight, bias, eps):
            with torch.no_grad():
                mean, rstd = x.mean(-1), (x.var(-1, unbiased=False) + eps).rsqrt()
                return (x - mean[:, None]) * rstd[:, None] * weight + bias, mean, rstd

        @staticmethod
        def layer_norm_bwd(dy, x, mean, rstd, weight, *need):
            with torch.no_grad():
                xhat, g = (x - mean[:, None]) * rstd[:, None], dy * weight
                dx = rstd[:, None] * (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True))
                return dx, (dy * xhat).sum(0), dy.sum(0)

    monkeypatch.setattr(autograd, "context", lambda device: Formulas)
    x = torch.randn(3, 8, requires_grad=True)
    w, b = torch.rand(8, requires_grad=True), torch.zeros(8, requires_grad=True)
    for loss in (lambda y: y.square().sum(), lambda y: (y * torch.arange(8.0)).sum()):      # dy has a graph; has none
        for of in (x, w):
            first = torch.autograd.grad(loss(autograd.layer_norm(x, w, b)), of, create_graph=True)[0]
            with pytest.raises(RuntimeError, match="differentiable once"):
                (first.square().sum() + x.sum()).backward()
    x.grad = None
    autograd.layer_norm(x, w, b).square().sum().backward()          # one derivative as ever
    assert torch.allclose(x.grad, torch.autograd.grad(torch.nn.functional.layer_norm(x, (8,), w, b).square().sum(), x)[0], atol=1e-4)


@pytest.fixture
def int8_modules(monkeypatch):
    """The modules of int8.py with the quantizer played by its formula, codes in rows of a multiple of 16 bytes."""
    from paper_2112_10769_b200 import int8

    class Formulas:
        @staticmethod
        def quant_int8_rows(w):
            codes = torch.zeros(w.shape[0], -(-w.shape[1] // 16) * 16, dtype=torch.int8)[:, :w.shape[1]]
            scale = w.abs().amax(1) / 127
            codes.copy_((w / scale[:, None]).round())
            return codes, scale

    monkeypatch.setattr(int8.autograd, "context", lambda device: Formulas)
    return int8


def test_the_modules_answer_as_of_their_making(int8_modules):
    # codes and scales are a snapshot of the weight, so the other parameters have to be one too
    lin, norm = torch.nn.Linear(40, 24), torch.nn.LayerNorm(40)
    bias = torch.zeros(2, 24)
    layers = int8_modules.Int8Linear.of(lin, norm=norm), int8_modules.Int8Experts(torch.randn(2, 24, 40), bias)
    before = [{k: v.clone() for k, v in layer.state_dict().items()} for layer in layers]
    with torch.no_grad():
        for p in (*lin.parameters(), *norm.parameters(), bias):
            p.add_(1)
    for layer, state in zip(layers, before):
        for k, v in layer.state_dict().items():
            assert torch.equal(v, state[k]), k


def rows_fit_the_products(codes):
    return codes.stride(-1) == 1 and all(s % 16 == 0 for s in codes.stride()[:-1]) and codes.data_ptr() % 16 == 0


@pytest.mark.parametrize("how", ["bfloat16", "half", "double", "clone", "pickle", "assign"])
def test_the_modules_can_be_moved_and_cast(int8_modules, how):
    # the calls read float32 scales and parameters, and codes whose rows start at multiples of 16 bytes: a cast, a move
    # (which packs rows of 40 codes tightly, like clone) and loaded tensors have to leave both
    import io
    from paper_2112_10769_b200 import autograd
    layers = (int8_modules.Int8Linear.of(torch.nn.Linear(40, 24), norm=torch.nn.LayerNorm(40)),
              int8_modules.Int8Experts(torch.randn(2, 24, 40), torch.randn(2, 24)), autograd.LayerNorm(40))
    for layer in layers:
        before = {k: v.clone() for k, v in layer.state_dict().items()}
        if how == "clone":
            layer._apply(lambda t: t.clone(memory_format=torch.contiguous_format))
        elif how == "pickle":
            file = io.BytesIO()
            torch.save(layer.state_dict(), file)
            file.seek(0)
            layer.load_state_dict(torch.load(file))
        elif how == "assign":
            layer.load_state_dict({k: v.contiguous() if v.dtype == torch.int8 else v.double() for k, v in before.items()}, assign=True)
        else:
            getattr(layer, how)()
        after = layer.state_dict()
        assert list(after) == list(before)
        for k, v in after.items():
            assert v.dtype == before[k].dtype and v.shape == before[k].shape and torch.equal(v, before[k]), k
            assert v.dtype != torch.int8 or rows_fit_the_products(v), k
        assert all(p.requires_grad for p in layer.parameters())
