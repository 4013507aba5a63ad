"""Cases, plain forms and exact values of the operators of a block that answers in 8 bits.

Operators (``x`` rows are tokens, ``W`` is ``[N, K]`` as in ``torch.nn.Linear``, codes are int8 in -127..127):

  norm_fwd   layer norm, forward: y, and the mean and 1/std of every row that the backward pass needs
  norm_bwd   layer norm, backward: dx, and the weight's and bias's gradients summed over all rows
  linear     tokens quantized with a scale each, times int8 weights with a scale for each output channel
  prenorm    layer norm, its result quantized with a scale for each token, times int8 weights (as above)
  experts    the product of ``linear`` with one weight for each expert; the rows of an expert follow one another

A plain form is elementary torch operations in 32 bits, rounded once at the end; ``exact`` is the definition in 64 bits.
Quantization of a row: scale = max|x| / 127, q = x * fl32(127 / max|x|) in binary32 rounded to the nearest
whole number, ties to even.
"""
import math

import torch

own = False

EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- cases --------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one token of a model that answers: nothing but latency
        {"name": "norm_fwd one token", "op": "norm_fwd", "rows": 1, "cols": 1024, "pad": 0, "dtype": "bf16"},
        # a training batch of the benchmark's Transformer layer (8192 tokens, width 1024), activations in 32 bits
        {"name": "norm_fwd batch", "op": "norm_fwd", "rows": 8192, "cols": 1024, "pad": 0, "dtype": "f32"},
        # odd width, rows cut out of a wider tensor: nothing is aligned
        {"name": "norm_bwd odd strided", "op": "norm_bwd", "rows": 4099, "cols": 771, "pad": 5, "dtype": "f32"},
        # a long training batch of a wide model
        {"name": "norm_bwd wide batch", "op": "norm_bwd", "rows": 16384, "cols": 4096, "pad": 0, "dtype": "bf16"},
        # one token through norm and projection
        {"name": "prenorm one token", "op": "prenorm", "rows": 1, "N": 4096, "K": 1024, "bias": True, "dtype": "bf16"},
        # a prompt of the benchmark's Transformer layer through norm and the feed-forward's first product
        {"name": "prenorm prompt", "op": "prenorm", "rows": 8192, "N": 4096, "K": 1024, "bias": True, "dtype": "bf16"},
        # a few requests answered side by side, one token each: the weights' bytes
        {"name": "linear few tokens", "op": "linear", "rows": 5, "N": 4096, "K": 4096, "bias": False, "dtype": "bf16"},
        # sizes that fit no tile, 32-bit activations
        {"name": "linear odd sizes", "op": "linear", "rows": 333, "N": 1537, "K": 1000, "bias": True, "dtype": "f32"},
        # a long prompt of a wide model: the tensor cores
        {"name": "linear long prompt", "op": "linear", "rows": 16384, "N": 4096, "K": 4096, "bias": False, "dtype": "bf16"},
        # requests answered side by side, two experts for each token: the weights of the experts that were chosen
        {"name": "experts few tokens", "op": "experts", "rows": 32, "E": 64, "N": 2048, "K": 1024, "skew": 0.5, "bias": False, "dtype": "bf16"},
        # a short prompt over many experts: a few odd rows each, some none
        {"name": "experts odd ragged", "op": "experts", "rows": 1003, "E": 60, "N": 1400, "K": 520, "skew": 1.0, "bias": True, "dtype": "f32"},
        # a long prompt, two experts for each token, some experts preferred
        {"name": "experts long prompt", "op": "experts", "rows": 16384, "E": 16, "N": 4096, "K": 2048, "skew": 0.5, "bias": False, "dtype": "bf16"},
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["norm_fwd", "norm_bwd", "prenorm", "linear", "linear", "experts", "experts"])
    dtype = rng.choice(["f32", "bf16"])
    if op in ("norm_fwd", "norm_bwd"):
        cols = log(16, 12288)
        if rng.random() < 0.5:
            cols = -(-cols // 64) * 64
        rows = log(1, min(65536, max(1, 16384 * 4096 // (2 if dtype == "f32" else 1) // cols)))
        return {"op": op, "rows": rows, "cols": cols, "pad": rng.choice([0, 0, 8, rng.randrange(1, 64)]), "dtype": dtype}
    N, K = log(64, 8192), log(64, 8192)
    if rng.random() < 0.5:
        N, K = -(-N // 64) * 64, -(-K // 64) * 64
    if op == "prenorm":
        rows, dtype = log(1, min(16384, 16384 * 4096 * 4096 // (N * K))), "bf16"
        return {"op": op, "rows": rows, "N": N, "K": K, "bias": rng.random() < 0.5, "dtype": dtype}
    if op == "linear":
        rows = log(1, min(16384, 16384 * 4096 * 4096 // (N * K)))
        return {"op": op, "rows": rows, "N": N, "K": K, "bias": rng.random() < 0.5, "dtype": dtype}
    N, K = min(N, 4096), min(K, 4096)
    E = log(2, min(128, max(2, (1 << 28) // (N * K))))
    rows = log(1, 16384)
    while rows > 1 and (rows * N * K > 16384 * 4096 * 2048 or min(rows, 64) * E * max(N, K) > 1 << 27):
        rows //= 2
    return {"op": op, "rows": rows, "E": E, "N": N, "K": K, "skew": rng.choice([0.0, 0.5, 1.0]), "bias": rng.random() < 0.5, "dtype": dtype}


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _tokens(rows, cols, pad, dtype, gen):
    """Activations as a trained model has them: rows of different size, and a few channels far above the others."""
    x = torch.randn(rows, cols + pad, device="cuda", generator=gen)
    x *= torch.exp(0.5 * torch.randn(rows, 1, device="cuda", generator=gen))
    x *= 1 + 9 * (torch.rand(cols + pad, device="cuda", generator=gen) < 0.005)
    return x.to(TYPES[dtype])[:, :cols]


def _weights(E, N, K, gen):
    """int8 codes [E, N, K] (rows start every multiple of 16 bytes) and the scale of each output channel [E, N]."""
    codes = torch.empty(E, N, -(-K // 16) * 16, dtype=torch.int8, device="cuda")
    scale = torch.empty(E, N, device="cuda")
    for e in range(E):
        w = torch.randn(N, codes.shape[2], device="cuda", generator=gen) * (K ** -0.5)
        w *= torch.exp(0.3 * torch.randn(N, 1, device="cuda", generator=gen))
        top = w.abs().amax(1, keepdim=True)
        codes[e] = (w * (127 / top)).round().to(torch.int8)
        scale[e] = top[:, 0] / 127
    return codes[:, :, :K], scale


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    s = dict(case)
    if case["op"] in ("norm_fwd", "norm_bwd"):
        rows, cols = case["rows"], case["cols"]
        s["x"] = _tokens(rows, cols, case["pad"], case["dtype"], gen)
        s["weight"] = 1 + 0.2 * torch.randn(cols, device="cuda", generator=gen)
        s["bias"] = 0.1 * torch.randn(cols, device="cuda", generator=gen)
        if case["op"] == "norm_bwd":
            s["dy"] = (1e-3 * torch.randn(rows, cols + case["pad"], device="cuda", generator=gen)).to(TYPES[case["dtype"]])[:, :cols]
            x = s["x"].double()
            mean = x.mean(1)
            s["mean"] = mean.float()
            s["rstd"] = ((x - mean[:, None]).square().mean(1) + EPS).rsqrt().float()
        return s
    E, N, K = case.get("E", 1), case["N"], case["K"]
    s["x"] = _tokens(case["rows"], K, 0, case["dtype"], gen)
    s["w"], s["w_scale"] = _weights(E, N, K, gen)
    s["w_bias"] = 0.1 * torch.randn(E, N, device="cuda", generator=gen) if case["bias"] else None
    if case["op"] == "experts":
        # a row's expert by popularity; the rows come sorted by expert, as a router hands them on
        popular = torch.arange(1, E + 1, device="cuda", dtype=torch.float32).pow(-case["skew"])
        popular = popular[torch.randperm(E, device="cuda", generator=gen)]
        s["expert"] = torch.multinomial(popular, case["rows"], replacement=True, generator=gen).sort().values
        counts = torch.bincount(s["expert"], minlength=E)
        s["offsets"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
        s["most"] = int(counts.max())
    else:
        s["w"], s["w_scale"] = s["w"][0], s["w_scale"][0]
        s["w_bias"] = s["w_bias"][0] if case["bias"] else None
        if case["op"] == "prenorm":
            s["weight"] = 1 + 0.2 * torch.randn(K, device="cuda", generator=gen)
            s["bias"] = 0.1 * torch.randn(K, device="cuda", generator=gen)
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------------
def _norm(x, weight, bias):
    x = x.float()
    mean = x.mean(1, keepdim=True)
    centred = x - mean
    rstd = (centred.square().mean(1, keepdim=True) + EPS).rsqrt()
    return centred * rstd * weight + bias, mean, rstd


def _norm_grad(x, dy, weight, mean, rstd):
    x, dy = x.float(), dy.float()
    xhat = (x - mean[:, None]) * rstd[:, None]
    g = dy * weight
    dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return dx, (dy * xhat).sum(0), dy.sum(0)


def _quantize(x):
    x = x.float()
    top = x.abs().amax(1, keepdim=True)
    q = (x * torch.where(top > 0, 127 / top, 0.0)).round()
    return q, top / 127


def _plain(s):
    op, x = s["op"], s["x"]
    if op == "norm_fwd":
        y, mean, rstd = _norm(x, s["weight"], s["bias"])
        return {"y": y.to(x.dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if op == "norm_bwd":
        dx, dweight, dbias = _norm_grad(x, s["dy"], s["weight"], s["mean"], s["rstd"])
        return {"dx": dx.to(x.dtype), "dweight": dweight, "dbias": dbias}
    if op == "experts":
        # the rows of every expert in a block of their own, padded to the longest, then one product for all of them
        q, scale = _quantize(x)
        E = s["w"].shape[0]
        at = torch.arange(x.shape[0], device=x.device) - s["offsets"][s["expert"]]
        block = q.new_zeros(E, s["most"], x.shape[1])
        block[s["expert"], at] = q
        z = torch.bmm(block, s["w"].float().transpose(1, 2))[s["expert"], at]
        z = z * scale * s["w_scale"][s["expert"]]
        z = z if s["w_bias"] is None else z + s["w_bias"][s["expert"]]
        return z.to(x.dtype)
    q, scale = _quantize(_norm(x, s["weight"], s["bias"])[0] if op == "prenorm" else x)
    z = (q @ s["w"].float().t()) * scale * s["w_scale"]
    z = z if s["w_bias"] is None else z + s["w_bias"]
    return z.to(x.dtype)


# ---- the framework's calls ------------------------------------------------------------------------------------------------
_lib = None


def _context(device):
    global _lib
    if _lib is None:
        from paper_2112_10769_b200 import autograd as _lib
    return _lib.context(device)


def _own(s):
    op, x = s["op"], s["x"]
    ctx = _context(x.device)
    if op == "norm_fwd":
        y, mean, rstd = ctx.layer_norm(x, s["weight"], s["bias"], EPS)
        return {"y": y, "mean": mean, "rstd": rstd}
    if op == "norm_bwd":
        dx, dweight, dbias = ctx.layer_norm_bwd(s["dy"], x, s["mean"], s["rstd"], s["weight"])
        return {"dx": dx, "dweight": dweight, "dbias": dbias}
    if op == "experts":
        return ctx.quant_int8_gemm_grouped(x, s["offsets"], s["w"], s["w_scale"], s["w_bias"])
    if op == "prenorm":
        return ctx.layer_norm_int8_gemm(x, s["weight"], s["bias"], EPS, s["w"], s["w_scale"], s["w_bias"])
    return ctx.quant_int8_gemm(x, s["w"], s["w_scale"], s["w_bias"])


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------
def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    rows = case["rows"]
    if case["op"] == "norm_fwd":
        cols = case["cols"]
        return {"bytes": 2 * size * rows * cols + 8 * cols + 8 * rows, "flops": 8 * rows * cols}
    if case["op"] == "norm_bwd":
        cols = case["cols"]
        return {"bytes": 3 * size * rows * cols + 12 * cols + 8 * rows, "flops": 13 * rows * cols}
    N, K = case["N"], case["K"]
    used = min(rows, case.get("E", 1))     # at most so many experts have rows
    small = used * N * (8 if case["bias"] else 4) + (8 * K if case["op"] == "prenorm" else 0) + 4 * case.get("E", 0)
    return {"bytes": size * rows * (N + K) + used * N * K + small, "flops": 2 * rows * N * K}


# ---- 64 bits ------------------------------------------------------------------------------------------------------------------
def _codes64(x):
    """The whole numbers of a row and its scale: 127 / max and its product with x are binary32, as the definition says."""
    if x.dtype != torch.float64:
        top = x.abs().amax(1, keepdim=True).double()
        factor = torch.where(top > 0, (127 / top).float().double(), torch.zeros_like(top))
        return (x.double() * factor).float().double().round(), top / 127
    top = x.abs().amax(1, keepdim=True)
    return (x * torch.where(top > 0, 127 / top, torch.zeros_like(top))).round(), top / 127


def exact(case, seed):
    s = prepare(case, seed)
    op, x = s["op"], s["x"]
    if op == "norm_bwd":
        # with xhat from the mean and 1/std that the call is given
        mean, rstd, w = (s[k].double() for k in ("mean", "rstd", "weight"))
        x, dy = x.double(), s["dy"].double()
        xhat = torch.addcmul(-(mean * rstd)[:, None], x, rstd[:, None])
        cols = x.shape[1]
        along, straight = (dy * xhat) @ w / cols, dy @ w / cols
        dx = (dy * w - straight[:, None] - along[:, None] * xhat) * rstd[:, None]
        return {"dx": dx, "dweight": torch.einsum("rc,rc->c", dy, xhat), "dbias": dy.sum(0)}
    if op in ("norm_fwd", "prenorm"):
        var, mean = torch.var_mean(x.double(), 1, unbiased=False, keepdim=True)
        std = torch.sqrt(var + EPS)
        y = (x.double() - mean) / std * s["weight"].double() + s["bias"].double()
        if op == "norm_fwd":
            return {"y": y, "mean": mean[:, 0], "rstd": 1 / std[:, 0]}
        x = y
    q, scale = _codes64(x)
    w, w_scale, w_bias = s["w"], s["w_scale"], s["w_bias"]
    if op != "experts":
        w, w_scale, w_bias = w[None], w_scale[None], None if w_bias is None else w_bias[None]
        ends = [0, x.shape[0]]
    else:
        ends = s["offsets"].tolist()
    z = torch.zeros(x.shape[0], w.shape[1], dtype=torch.float64, device=x.device)
    for e in range(w.shape[0]):
        a, b = ends[e], ends[e + 1]
        if b > a:
            z[a:b] = torch.einsum("tk,nk->tn", q[a:b] * scale[a:b], w[e].double() * w_scale[e].double()[:, None])
            if w_bias is not None:
                z[a:b] += w_bias[e].double()
    return z
