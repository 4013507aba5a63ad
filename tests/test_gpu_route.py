"""Expert routing against the definition in 64 bits.  Choices are exact; weights are within 16 half steps of binary32 (an exponential of 2 ulp,
its argument's rounding, a sum over the experts in a tree, a quotient, a product); gradients within the same of the sum of their terms'
magnitudes, half a step of the logits' type more."""
import math

import pytest
import torch

from paper_2112_10769_b200 import binding, experts

pytestmark = pytest.mark.gpu
INF = math.inf


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def scores(x, score):
    if score == "sigmoid":
        return torch.sigmoid(x)
    top = x.amax(1, keepdim=True)
    p = torch.exp(x - torch.where(top == -INF, 0.0, top))
    return p / p.sum(1, keepdim=True).clamp_min(1e-300)


def reference(x, k, score="softmax", bias=None, groups=1, top_groups=1, group_top=2, renormalize=True, scale=1.0):
    """(experts, weights) of every row, in 64 bits: differentiable in x."""
    x = x.double()
    T, E = x.shape
    p = scores(x, score)
    with torch.no_grad():
        c = x.clone() if bias is None and groups == 1 else p.clone() if bias is None else p + bias.double()
        c[x == -INF] = -INF
        if groups > 1:
            best = c.view(T, groups, E // groups).sort(2, descending=True).values[:, :, :group_top]
            value = best[:, :, 0] + (torch.where(best[:, :, 1] == -INF, 0.0, best[:, :, 1]) if best.shape[2] > 1 else 0.0)
            stay = torch.sort(value, dim=1, descending=True, stable=True).indices[:, :top_groups]
            keep = torch.zeros(T, groups, dtype=torch.bool, device=x.device).scatter_(1, stay, True)
            c = torch.where(keep.repeat_interleave(E // groups, 1), c, -INF)
        value, chosen = torch.sort(c, dim=1, descending=True, stable=True)
        chosen = torch.where(value[:, :k] == -INF, -1, chosen[:, :k])
    w = torch.where(chosen < 0, 0.0, p.gather(1, chosen.clamp_min(0)))
    if renormalize:
        w = w / w.sum(1, keepdim=True).clamp_min(1e-300)
    return chosen.to(torch.int32), w * scale


def logits(T, E, dtype, kind, seed=0):
    g = torch.Generator("cuda").manual_seed(seed + 31 * T + E)
    x = 1.5 * torch.randn(T, E, device="cuda", generator=g)
    if kind == "ties":
        x = (2 * x).round() / 2
    if kind == "masked":
        x[torch.rand(T, E, device="cuda", generator=g) < 0.6] = -INF
        x[T // 2:] = -INF
    if kind == "equal":
        x[:] = 0.25
    if kind == "close":                                     # values that binary32 does not tell apart, and their biases
        x = 0.5 + 1e-7 * torch.randint(-3, 4, (T, E), device="cuda", generator=g)
    return x.to(dtype)


SHAPES = [(1, 1, 1, 1, 1), (3, 8, 2, 1, 1), (1, 256, 8, 8, 4), (500, 256, 8, 8, 4), (70, 60, 4, 1, 1), (33, 64, 6, 8, 3), (40, 160, 6, 8, 3), (9, 1024, 32, 1, 1),
          (17, 1000, 9, 8, 2), (5, 32, 32, 1, 1), (64, 12, 3, 4, 2), (20, 33, 5, 1, 1), (100, 128, 16, 16, 16), (31, 512, 8, 4, 2), (50, 64, 2, 32, 1), (11, 97, 12, 1, 1)]


@pytest.mark.parametrize("T,E,k,groups,top_groups", SHAPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("kind", ["plain", "ties", "masked", "equal", "close"])
def test_choice_and_weights(ctx, T, E, k, groups, top_groups, score, kind):
    g = torch.Generator("cuda").manual_seed(T + E)
    for dtype in (torch.float32, torch.bfloat16):
        x = logits(T, E, dtype, kind)
        for bias in (None, 0.05 * torch.randn(E, device="cuda", generator=g), torch.zeros(E, device="cuda")):
            if kind == "close" and bias is not None:
                bias = bias * 1e-6
            for renormalize, group_top in ((True, 2), (False, 1)):
                form = dict(score=score, bias=bias, groups=groups, top_groups=top_groups, group_top=group_top, renormalize=renormalize, scale=2.5)
                e, w = ctx.route(x, k, **form)
                we, ww = reference(x, k, **form)
                assert torch.equal(e, we)
                assert ((w.double() - ww).abs() <= 16 * 2.0 ** -24 * ww).all()
                assert torch.equal(ctx.route(x, k, **form)[1], w)
    assert ctx.status() == 0


def test_many_rows_with_values_next_to_a_border(ctx):
    # enough rows that some places and some groups are closer than binary32 tells
    for score, dtype in (("sigmoid", torch.float32), ("softmax", torch.float32), ("softmax", torch.bfloat16)):
        x = logits(30000, 256, dtype, "plain", 5)
        bias = 0.05 * torch.randn(256, device="cuda")
        for form in (dict(bias=bias, groups=8, top_groups=4), dict(bias=bias), dict(groups=8, top_groups=4), dict()):
            assert torch.equal(ctx.route(x, 8, score=score, **form)[0], reference(x, 8, score=score, **form)[0])


@pytest.mark.parametrize("pad,shift", [(0, 0), (4, 0), (3, 1), (0, 1)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_a_wider_tensor(ctx, dtype, pad, shift):
    for T, E, k in ((5, 64, 4), (40, 256, 8), (7, 100, 3)):
        base = logits(T, E + pad + shift, dtype, "plain")
        x = base[:, shift:shift + E]
        e, w = ctx.route(x, k)
        we, ww = ctx.route(x.clone(), k)
        assert torch.equal(e, we) and torch.equal(w, ww)
        dw = torch.randn(T, k, device="cuda")
        for renormalize in (True, False):
            assert torch.equal(ctx.route_bwd(dw, x, e, renormalize=renormalize), ctx.route_bwd(dw, x.clone(), e, renormalize=renormalize))


def test_rows_with_nan_or_infinity(ctx):
    x = logits(6, 40, torch.float32, "plain")
    want = ctx.route(x, 3)
    bad = x.clone()
    bad[1, 7], bad[3, 0] = math.nan, INF
    for form in (dict(), dict(score="sigmoid"), dict(bias=torch.zeros(40, device="cuda")), dict(groups=4, top_groups=2)):
        e, w = ctx.route(bad, 3, **form)
        assert ctx.status() == binding.STATUS_NONFINITE
        assert (e[[1, 3]] == -1).all() and torch.isnan(w[[1, 3]]).all()
        good = [0, 2, 4, 5]
        ge, gw = ctx.route(x[good], 3, **form)
        assert torch.equal(e[good], ge) and torch.equal(w[good], gw) and ctx.status() == 0
    bias = torch.zeros(40, device="cuda")
    bias[5] = -INF                                          # never chosen
    x[:, 5] = 50.0
    assert (ctx.route(x, 3, bias=bias)[0] != 5).all() and ctx.status() == 0
    bias[5] = math.nan
    e, w = ctx.route(x, 3, bias=bias)
    assert (e == -1).all() and torch.isnan(w).all() and ctx.status() == binding.STATUS_NONFINITE
    assert torch.equal(e, torch.full_like(e, -1)) and want[0].shape == e.shape


@pytest.mark.parametrize("T,E,k,groups,top_groups", SHAPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_gradient(ctx, T, E, k, groups, top_groups, score):
    for kind in ("plain", "masked"):
        for dtype in (torch.float32, torch.bfloat16):
            for renormalize in (True, False):
                x = logits(T, E, dtype, kind).requires_grad_()
                form = dict(score=score, groups=groups, top_groups=top_groups, renormalize=renormalize, scale=1.7)
                chosen, w = experts.route(x, k, **form)
                dw = torch.randn(T, k, device="cuda")
                (w * dw).sum().backward()
                live = (x.detach() > -INF).any(1)           # (the reference's softmax has no gradient where nothing is left)
                x64 = x.detach().double().requires_grad_()
                (reference(x64, k, **form)[1] * dw.double()).sum().backward()
                want = torch.where(live[:, None] & (x64 > -INF), x64.grad, 0.0).nan_to_num(0.0)
                # the terms of a row's gradient: its weights and their sum, times at most the largest of dw, twice
                size = 4 * 1.7 * dw.abs().amax(1, keepdim=True).double() * (scores(x.detach().double(), score).nan_to_num(0.0) + want.abs())
                share = torch.zeros_like(size).scatter_add_(1, chosen.clamp_min(0).long(), torch.where(chosen < 0, 0.0, w.detach().double()))
                bound = 16 * 2.0 ** -24 * (size + 4 * share * dw.abs().amax(1, keepdim=True))
                got = x.grad.double()
                bound = bound + (2.0 ** -8 * (want.abs() + bound) if dtype == torch.bfloat16 else 0.0)
                assert ((got - want).abs() <= bound).all()


def test_gradient_against_differences(ctx):
    x = logits(4, 12, torch.float32, "plain")
    dw = torch.randn(4, 3, device="cuda")
    for score in ("softmax", "sigmoid"):
        for renormalize in (True, False):
            chosen, _ = ctx.route(x, 3, score=score, renormalize=renormalize)
            def f(v):                                       # with the choice held
                p = scores(v.double(), score).gather(1, chosen.long())
                return ((p / p.sum(1, keepdim=True) if renormalize else p) * dw.double()).sum().item()
            grad = ctx.route_bwd(dw, x, chosen, score=score, renormalize=renormalize)
            for t, e in ((0, 0), (1, int(chosen[1, 0])), (2, int(chosen[2, 2])), (3, 11)):
                step = torch.zeros_like(x)
                step[t, e] = 2.0 ** -8
                # the third difference's share of a step of 2^-8 is below 2^-16 of the largest dw
                assert abs((f(x + step) - f(x - step)) / 2.0 ** -7 - grad[t, e].item()) < 4 * 2.0 ** -16 * dw.abs().max().item()


def test_gradient_of_an_expert_in_several_places(ctx):
    x = logits(3, 8, torch.float32, "plain")
    chosen = torch.tensor([[2, 2, 5], [1, -1, 1], [-1, 99, -7]], dtype=torch.int32, device="cuda")
    dw = torch.randn(3, 3, device="cuda")
    for score in ("softmax", "sigmoid"):
        for renormalize in (True, False):
            x64 = x.double().requires_grad_()
            there = (chosen >= 0) & (chosen < 8)
            p = torch.where(there, scores(x64, score).gather(1, chosen.clamp(0, 7).long()), 0.0)
            w = p / p.sum(1, keepdim=True).clamp_min(1e-300) if renormalize else p
            (w * dw.double()).sum().backward()
            got = ctx.route_bwd(dw, x, chosen, score=score, renormalize=renormalize)
            assert ((got.double() - x64.grad).abs() <= 32 * 2.0 ** -24 * 4 * dw.abs().max()).all()


def test_second_derivative_raises(ctx):
    x = logits(4, 8, torch.float32, "plain").requires_grad_()
    _, w = experts.route(x, 2, renormalize=False)
    grad, = torch.autograd.grad((w * w).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="differentiable once"):
        grad.sum().backward()


def test_refusals(ctx):
    x = logits(4, 24, torch.float32, "plain")
    for call in (lambda: ctx.route(x, 0), lambda: ctx.route(x, 25), lambda: ctx.route(x, 2, score="tanh"), lambda: ctx.route(x.half(), 2), lambda: ctx.route(x.cpu(), 2),
                 lambda: ctx.route(x, 2, bias=torch.zeros(23, device="cuda")), lambda: ctx.route(x, 2, bias=torch.zeros(24, device="cuda").half()),
                 lambda: ctx.route_bwd(torch.zeros(4, 3, device="cuda"), x, torch.zeros(4, 2, dtype=torch.int32, device="cuda")),
                 lambda: ctx.route_bwd(torch.zeros(4, 2, device="cuda"), x, torch.zeros(4, 2, dtype=torch.int64, device="cuda")),
                 lambda: ctx.route_bwd(torch.zeros(3, 2, device="cuda"), x, torch.zeros(3, 2, dtype=torch.int32, device="cuda"))):
        with pytest.raises(TypeError):
            call()
    wide = torch.zeros(2, 1025, device="cuda")
    for call in (lambda: ctx.route(x, 2, groups=3, top_groups=2), lambda: ctx.route(x, 2, groups=16, top_groups=2), lambda: ctx.route(x, 2, groups=4, top_groups=5),
                 lambda: ctx.route(x, 13, groups=4, top_groups=2), lambda: ctx.route(x, 2, group_top=3), lambda: ctx.route(wide, 2), lambda: ctx.route(wide[:, :64], 33),
                 lambda: ctx.route(x, 2, groups=4, top_groups=0)):
        with pytest.raises(binding.LuqError) as e:
            call()
        assert e.value.code == binding.ERR_ARG
    assert ctx.route(x[:0], 2)[0].shape == (0, 2) and ctx.status() == 0


# many rows, so that groups, places and whole rows that binary32 leaves open are among them; as many places as lanes have a row; rows
# that share a warp with open ones
@pytest.mark.parametrize("T,E,k,groups,top_groups,kind", [(20000, 512, 8, 4, 2, "plain"), (20000, 160, 6, 8, 3, "plain"), (6000, 1000, 32, 8, 4, "plain"), (20000, 64, 8, 8, 4, "plain"),
                                                          (3001, 64, 8, 8, 5, "close"), (3001, 128, 16, 4, 2, "close"), (2000, 1024, 32, 32, 20, "close"), (3001, 60, 8, 1, 1, "close")])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_many_rows_left_open(ctx, T, E, k, groups, top_groups, kind, score):
    g = torch.Generator("cuda").manual_seed(T + E)
    bias = (0.05 if kind == "plain" else 5e-8) * torch.randn(E, device="cuda", generator=g)
    x = logits(T, E, torch.float32, kind, 9)
    if kind == "close":                                     # every other row is clear of it all
        x[1::2] += 0.01 * torch.randperm(E, device="cuda", generator=g)
    for group_top in (1, 2):
        for b in (bias, None):
            form = dict(score=score, bias=b, groups=groups, top_groups=top_groups, group_top=group_top)
            assert torch.equal(ctx.route(x, k, **form)[0], reference(x, k, **form)[0])
    assert ctx.status() == 0
