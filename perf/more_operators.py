"""Cases, plain forms and exact values of the operators of a layer of experts, and of products in 4-bit floating point.

Operators (rows of ``x`` are tokens, ``W`` is ``[N, K]`` as in ``torch.nn.Linear``, k experts are chosen for each token):

  route         scores of all experts -> the k experts of every token and their weights
  route_bwd     gradient of the weights -> gradient of the logits
  dispatch      experts of every token -> offsets of the experts, position of every copy; tokens copied to their positions
  combine       weighted sum of a token's k results, added to a residual
  combine_bwd   gradients of the results and of the weights
  linear        tokens quantized to blocks of 4-bit numbers, times weights of that form
  experts       dispatch and the product of ``linear`` with one weight for each expert, in one call

4-bit numbers are e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, rounded to nearest, ties to the even code.  A row's
blocks have a scale each.  Blocks of 32: 2^(floor(log2 max|block|) - 2).  Blocks of 16: an e4m3 number, and a scale g for the row;
every step in binary32: g = max|row| / 2688, s = e4m3(max|block| / (6 g)), q = e2m1(x * (1 / (s g))).

A plain form is elementary torch operations in 32 bits, rounded once at the end (experts are chosen by values in 64: the
k-th and the next may lie next to one another); ``exact`` is the definition in 64 bits.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---- cases --------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one token of a model that answers, many experts in groups, bias for balance: nothing but latency
        {"name": "route one token", "op": "route", "T": 1, "E": 256, "k": 8, "score": "sigmoid", "bias": True, "groups": 8, "top_groups": 4, "renorm": True, "padded": 0, "dtype": "f32"},
        # a long prompt, the same choice
        {"name": "route prompt", "op": "route", "T": 16384, "E": 256, "k": 8, "score": "sigmoid", "bias": True, "groups": 8, "top_groups": 4, "renorm": True, "padded": 0, "dtype": "f32"},
        # a training batch of a model with few experts and softmax scores, padded at its end
        {"name": "route_bwd batch", "op": "route_bwd", "T": 32768, "E": 60, "k": 4, "score": "softmax", "bias": False, "groups": 1, "top_groups": 1, "renorm": False, "padded": 1001, "dtype": "f32"},
        # requests answered side by side, one token each
        {"name": "dispatch few tokens", "op": "dispatch", "T": 48, "cols": 1024, "E": 64, "k": 2, "skew": 0.5, "padded": 0, "dtype": "bf16"},
        # a training batch of the benchmark's Transformer layer (8192 tokens, width 1024), eight experts of many for each token
        {"name": "dispatch batch", "op": "dispatch", "T": 8192, "cols": 1024, "E": 128, "k": 8, "skew": 0.5, "padded": 300, "dtype": "bf16"},
        # the same batch on its way back, added to the stream that went around the experts
        {"name": "combine batch", "op": "combine", "T": 8192, "cols": 1024, "k": 8, "residual": True, "padded": 300, "dtype": "bf16"},
        # odd width, 32 bits: nothing is aligned
        {"name": "combine_bwd odd", "op": "combine_bwd", "T": 4099, "cols": 771, "k": 3, "residual": False, "padded": 57, "dtype": "f32"},
        # one token through a projection of a wide model: the weights' bytes
        {"name": "linear one token", "op": "linear", "rows": 1, "N": 4096, "K": 4096, "block": 16, "bias": False, "dtype": "bf16"},
        # sizes that fit no tile, 32-bit activations, power-of-two scales
        {"name": "linear odd sizes", "op": "linear", "rows": 333, "N": 1537, "K": 1000, "block": 32, "bias": True, "dtype": "f32"},
        # a long prompt of a wide model: the tensor cores
        {"name": "linear long prompt", "op": "linear", "rows": 16384, "N": 4096, "K": 4096, "block": 16, "bias": False, "dtype": "bf16"},
        # requests answered side by side, two experts for each token: the weights of the experts that were chosen
        {"name": "experts few tokens", "op": "experts", "T": 32, "E": 64, "k": 2, "N": 2048, "K": 1024, "skew": 0.5, "block": 16, "bias": False, "dtype": "bf16"},
        # a long prompt, two experts for each token, some preferred
        {"name": "experts long prompt", "op": "experts", "T": 8192, "E": 16, "k": 2, "N": 4096, "K": 2048, "skew": 0.5, "block": 32, "bias": True, "dtype": "bf16"},
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["route", "route_bwd", "dispatch", "combine", "combine_bwd", "linear", "linear", "experts", "experts"])
    dtype = rng.choice(["f32", "bf16"])
    size = 4 if dtype == "f32" else 2
    if op in ("route", "route_bwd"):
        groups = rng.choice([1, 1, 2, 4, 8])
        each = log(max(2, 8 // groups), 512 // groups)
        top_groups = rng.randrange((groups + 1) // 2, groups + 1)
        E, T = groups * each, log(1, 32768)
        while T * E > 16384 * 256:
            T //= 2
        return {"op": op, "T": T, "E": E, "k": rng.randrange(1, min(8, top_groups * each) + 1), "score": rng.choice(["softmax", "sigmoid"]),
                "bias": rng.random() < 0.5, "groups": groups, "top_groups": top_groups, "renorm": rng.random() < 0.5,
                "padded": rng.choice([0, T // 20]), "dtype": dtype}
    k = rng.randrange(1, 9)
    if op in ("dispatch", "combine", "combine_bwd"):
        cols = log(16, 8192)
        if rng.random() < 0.5:
            cols = -(-cols // 64) * 64
        T = log(1, max(1, min(16384, 8192 * 1024 * 8 * 2 // (size * k * cols))))
        case = {"op": op, "T": T, "cols": cols, "k": k, "padded": rng.choice([0, T // 20]), "dtype": dtype}
        if op == "dispatch":
            case.update(E=log(max(2, k), 512), skew=rng.choice([0.0, 0.5, 1.0]))
        else:
            case.update(residual=op == "combine" and rng.random() < 0.5)
        return case
    N, K = log(64, 8192), log(64, 8192)
    if rng.random() < 0.5:
        N, K = -(-N // 64) * 64, -(-K // 64) * 64
    block = rng.choice([16, 32])
    if op == "linear":
        rows = log(1, min(16384, 16384 * 4096 * 4096 // (N * K)))
        return {"op": op, "rows": rows, "N": N, "K": K, "block": block, "bias": rng.random() < 0.5, "dtype": dtype}
    N, K = min(N, 4096), min(K, 4096)
    E = log(2, min(128, max(2, (1 << 28) // (N * K))))
    k = min(k, E)
    T = log(1, 8192)
    while T > 1 and (T * k * N * K > 16384 * 4096 * 2048 or min(T * k, 64) * E * max(N, K) > 1 << 27):
        T //= 2
    return {"op": op, "T": T, "E": E, "k": k, "N": N, "K": K, "skew": rng.choice([0.0, 0.5, 1.0]), "block": block,
            "bias": rng.random() < 0.5, "dtype": dtype}


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _tokens(rows, cols, dtype, gen):
    """Activations as a trained model has them: rows of different size, and a few channels far above the others."""
    x = torch.randn(rows, cols, device="cuda", generator=gen)
    x *= torch.exp(0.5 * torch.randn(rows, 1, device="cuda", generator=gen))
    x *= 1 + 9 * (torch.rand(cols, device="cuda", generator=gen) < 0.005)
    return x.to(TYPES[dtype])


def _choice(T, E, k, skew, padded, gen):
    """k different experts for every token, some preferred; -1 for the tokens that pad the batch."""
    popular = torch.arange(1, E + 1, device="cuda", dtype=torch.float32).pow(-skew)
    popular = popular[torch.randperm(E, device="cuda", generator=gen)]
    # the k largest of log(popularity) + Gumbel noise: a draw without replacement
    noise = -torch.log(-torch.log(torch.rand(T, E, device="cuda", generator=gen).clamp(1e-9, 1 - 1e-6)))
    experts = (popular.log() + noise).topk(k, 1).indices.to(torch.int32)
    experts[T - padded:] = -1
    return experts


def _positions(experts, E):
    """Offsets [E + 1] and positions [T, k]: copies sorted by expert, in the tokens' order within one."""
    flat = experts.flatten().long()
    key = torch.where(flat < 0, E, flat)
    order = torch.sort(key, stable=True).indices
    position = torch.empty_like(order)
    position[order] = torch.arange(order.numel(), device=order.device)
    position[flat < 0] = -1
    counts = torch.bincount(key, minlength=E + 1)[:E]
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
    return offsets, position.view(experts.shape).to(torch.int32)


def _weights(E, N, K, block, gen):
    """Packed codes [E, N, ceil(K / 2)] (the lower half of a byte is the earlier number; rows start every multiple of 16
    bytes), the blocks' scales as bytes [E, N, ceil(K / block)], the rows' scales [E, N] (blocks of 16)."""
    blocks = -(-K // block)
    codes = torch.zeros(E, N, -(-K // 32) * 16, dtype=torch.uint8, device="cuda")
    scale = torch.empty(E, N, blocks, dtype=torch.uint8, device="cuda")
    row = torch.empty(E, N, device="cuda") if block == 16 else None
    for e in range(E):
        w = torch.zeros(N, blocks * block, device="cuda")
        w[:, :K] = torch.randn(N, K, device="cuda", generator=gen) * (K ** -0.5)
        w *= torch.exp(0.3 * torch.randn(N, 1, device="cuda", generator=gen))
        q, s, g = _quantize(w, block)
        q = q.view(N, -1)
        index = torch.bucketize(q.abs(), torch.tensor(LEVELS, device="cuda")) + 8 * (q < 0)
        index = torch.nn.functional.pad(index, (0, 2 * codes.shape[2] - index.shape[1]))
        codes[e] = (index[:, 0::2] + 16 * index[:, 1::2]).to(torch.uint8)
        if block == 16:
            scale[e] = s.to(torch.float8_e4m3fn).view(torch.uint8)
            row[e] = g
        else:
            scale[e] = (torch.frexp(s).exponent + 126).to(torch.uint8)
    return codes[:, :, :(K + 1) // 2], scale, row


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    s, op = dict(case), case["op"]
    if op in ("route", "route_bwd"):
        T, E = case["T"], case["E"]
        x = 1.5 * torch.randn(T, E, device="cuda", generator=gen) + 0.5 * torch.randn(E, device="cuda", generator=gen)
        x[T - case["padded"]:] = -math.inf
        s["x"] = x.to(TYPES[case["dtype"]])
        s["balance"] = 0.05 * torch.randn(E, device="cuda", generator=gen) if case["bias"] else None
        if op == "route_bwd":
            s["experts"] = _chosen(s)[0]
            s["dweights"] = 1e-3 * torch.randn(T, case["k"], device="cuda", generator=gen)
        return s
    if op in ("dispatch", "combine", "combine_bwd"):
        T, cols, k = case["T"], case["cols"], case["k"]
        s["experts"] = _choice(T, case.get("E", max(8, k)), k, case.get("skew", 0.5), case["padded"], gen)
        if op == "dispatch":
            s["x"] = _tokens(T, cols, case["dtype"], gen)
            return s
        s["offsets"], s["position"] = _positions(s["experts"], max(8, k))
        s["y"] = _tokens(T * k, cols, case["dtype"], gen)
        s["weights"] = torch.rand(T, k, device="cuda", generator=gen).add_(0.1)
        s["weights"] /= s["weights"].sum(1, keepdim=True)
        s["res"] = _tokens(T, cols, case["dtype"], gen) if case["residual"] else None
        if op == "combine_bwd":
            s["dout"] = (1e-3 * torch.randn(T, cols, device="cuda", generator=gen)).to(TYPES[case["dtype"]])
        return s
    E, N, K, block = case.get("E", 1), case["N"], case["K"], case["block"]
    s["x"] = _tokens(case["rows"] if op == "linear" else case["T"], K, case["dtype"], gen)
    s["w"], s["w_scale"], s["w_row"] = _weights(E, N, K, block, gen)
    s["w_bias"] = 0.1 * torch.randn(E, N, device="cuda", generator=gen) if case["bias"] else None
    if op == "experts":
        s["experts"] = _choice(case["T"], E, case["k"], case["skew"], 0, gen)
        s["offsets"], s["position"] = _positions(s["experts"], E)
        s["most"] = int((s["offsets"][1:] - s["offsets"][:-1]).max())
    else:
        s["w"], s["w_scale"] = s["w"][0], s["w_scale"][0]
        s["w_row"] = None if s["w_row"] is None else s["w_row"][0]
        s["w_bias"] = s["w_bias"][0] if case["bias"] else None
    if own:
        # the scales as the tensor cores read them: laid out once, as the framework's modules keep them
        from paper_2112_10769_b200 import e2m1
        s["w_tiles"] = e2m1.scale_tiles(s["w_scale"], block)
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------------
def _chosen(s):
    """experts [T, k] (-1: none was left) and the scores of all experts, in 64 bits."""
    x = s["x"].double()
    T, E = x.shape
    if s["score"] == "sigmoid":
        score = torch.sigmoid(x)
    else:
        top = x.amax(1, keepdim=True)
        p = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
        score = p / p.sum(1, keepdim=True).clamp_min(1e-300)
    c = x if s["balance"] is None and s["groups"] == 1 else score if s["balance"] is None else score + s["balance"].double()
    c = torch.where(x == -math.inf, x, c)
    G = s["groups"]
    if G > 1:
        best = c.view(T, G, E // G).sort(2, descending=True).values[:, :, :2]
        value = torch.where(best[:, :, 1:] == -math.inf, best[:, :, :1], best.sum(2, keepdim=True))[:, :, 0] if best.shape[2] > 1 else best[:, :, 0]
        stay = torch.sort(value, dim=1, descending=True, stable=True).indices[:, :s["top_groups"]]
        keep = torch.zeros_like(value, dtype=torch.bool).scatter_(1, stay, True)
        c = torch.where(keep.repeat_interleave(E // G, 1), c, -math.inf)
    value, index = torch.sort(c, dim=1, descending=True, stable=True)
    value, index = value[:, :s["k"]], index[:, :s["k"]]
    return torch.where(value == -math.inf, -1, index).to(torch.int32), score


def _route(s):
    experts, score = _chosen(s)
    w = torch.where(experts < 0, 0.0, score.gather(1, experts.clamp_min(0).long()))
    if s["renorm"]:
        w = w / w.sum(1, keepdim=True).clamp_min(1e-300)
    return {"experts": experts, "weights": w.float()}


def _route_bwd(s):
    x, experts, dw = s["x"].float(), s["experts"].long(), s["dweights"]
    there = experts >= 0
    if s["score"] == "sigmoid":
        p = torch.sigmoid(x)
    else:
        top = x.amax(1, keepdim=True)
        p = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
        p = p / p.sum(1, keepdim=True).clamp_min(1e-30)
    chosen = torch.where(there, p.gather(1, experts.clamp_min(0)), 0.0)
    dw = torch.where(there, dw, 0.0)
    if s["renorm"]:
        total = chosen.sum(1, keepdim=True).clamp_min(1e-30)
        dw = (dw - (dw * chosen).sum(1, keepdim=True) / total) / total
    dp = torch.zeros_like(p).scatter_add_(1, experts.clamp_min(0), torch.where(there, dw, 0.0))
    if s["score"] == "sigmoid":
        dx = dp * p * (1 - p)
    else:
        dx = p * (dp - (dw * chosen).sum(1, keepdim=True))
    return dx.to(s["x"].dtype)


def _dispatch(s):
    offsets, position = _positions(s["experts"], s["E"])
    T, k = position.shape
    rows = torch.zeros(T * k, s["cols"], dtype=s["x"].dtype, device="cuda")
    to = position.flatten().long()
    token = torch.arange(T, device="cuda").repeat_interleave(k)
    rows[to[to >= 0]] = s["x"][token[to >= 0]]
    return {"rows": rows, "offsets": offsets, "position": position}


def _combine(s):
    position = s["position"].long()
    y = s["y"][position.clamp_min(0)].float() * torch.where(position >= 0, s["weights"], 0.0)[:, :, None]
    out = y.sum(1)
    out = out if s["res"] is None else out + s["res"].float()
    return out.to(s["y"].dtype)


def _combine_bwd(s):
    position, dout = s["position"].long(), s["dout"].float()
    there = position >= 0
    dw = torch.where(there, (s["y"][position.clamp_min(0)].float() * dout[:, None, :]).sum(2), 0.0)
    dy = torch.zeros_like(s["y"])
    dy[position[there]] = (s["weights"][:, :, None] * dout[:, None, :])[there].to(dy.dtype)
    return {"dy": dy, "dweights": dw}


def _round_e2m1(v):
    """The nearest of LEVELS with the sign of v, ties to the even code."""
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.copysign((a / step).round().mul(step).clamp_max(6.0), v)


def _quantize(x, block):
    """Values of the 4-bit numbers [rows, blocks, block], the blocks' scales [rows, blocks] and the rows' [rows] (blocks of 16)."""
    x = x.float()
    rows, cols = x.shape
    blocks = -(-cols // block)
    if cols % block:
        x = torch.nn.functional.pad(x, (0, blocks * block - cols))
    x = x.view(rows, blocks, block)
    top = x.abs().amax(2)
    if block == 32:
        s = torch.ldexp(torch.ones_like(top, dtype=torch.float64), torch.frexp(top).exponent - 3)
        s = torch.where(top > 0, s, 2.0 ** -127).clamp_min(2.0 ** -127)
        return _round_e2m1((x / s[:, :, None]).float()), s.float(), None
    g = torch.div(top.amax(1), torch.full_like(top[:, 0], 2688.0))
    six = g * 6.0
    s = torch.where(six[:, None] > 0, torch.div(top, six[:, None]), 0.0).to(torch.float8_e4m3fn).float()
    r = torch.where(s > 0, torch.div(torch.ones_like(s), s * g[:, None]), 0.0)
    return _round_e2m1(x * r[:, :, None]), s, g


def _weight_values(s, E, N, K, block):
    """The weights' values without the rows' scales, [E, N, K]."""
    codes = s["w"].reshape(E, N, -1)
    index = torch.stack([codes & 15, codes >> 4], 3).view(E, N, -1)[:, :, :K].long()
    levels = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device="cuda")
    scale = s["w_scale"].reshape(E, N, -1)
    scale = scale.view(torch.float8_e4m3fn).float() if block == 16 else torch.exp2(scale.float() - 127)
    return levels[index] * scale.repeat_interleave(block, 2)[:, :, :K]


def _product(s):
    x, N, K, block = s["x"], s["N"], s["K"], s["block"]
    q, scale, row = _quantize(x, block)
    q = (q * scale[:, :, None]).view(x.shape[0], -1)[:, :K]
    if s["op"] == "linear":
        z = q @ _weight_values(s, 1, N, K, block)[0].t()
        if block == 16:
            z = z * row[:, None] * s["w_row"]
        z = z if s["w_bias"] is None else z + s["w_bias"]
        return z.to(x.dtype)
    # the rows of every expert in a block of their own, padded to the longest, then one product for all of them
    E, T, k = s["E"], s["T"], s["k"]
    to = s["position"].flatten().long()
    token = torch.empty_like(to)
    token[to] = torch.arange(T, device="cuda").repeat_interleave(k)
    expert = torch.empty_like(to)
    expert[to] = s["experts"].flatten().long()
    at = torch.arange(T * k, device="cuda") - s["offsets"][expert]
    padded = q.new_zeros(E, s["most"], K)
    padded[expert, at] = q[token]
    z = torch.bmm(padded, _weight_values(s, E, N, K, block).transpose(1, 2))[expert, at]
    if block == 16:
        z = z * row[token][:, None] * s["w_row"][expert]
    z = z if s["w_bias"] is None else z + s["w_bias"][expert]
    return z.to(x.dtype)


def _plain(s):
    return {"route": _route, "route_bwd": _route_bwd, "dispatch": _dispatch, "combine": _combine, "combine_bwd": _combine_bwd,
            "linear": _product, "experts": _product}[s["op"]](s)


# ---- the framework's calls ------------------------------------------------------------------------------------------------
_lib = None


def _context(device):
    global _lib
    if _lib is None:
        from paper_2112_10769_b200 import autograd as _lib
    return _lib.context(device)


def _own(s):
    op = s["op"]
    ctx = _context(s["y"].device if "y" in s else s["x"].device)
    if op == "route":
        experts, weights = ctx.route(s["x"], s["k"], score=s["score"], bias=s["balance"], groups=s["groups"], top_groups=s["top_groups"],
                                     renormalize=s["renorm"])
        return {"experts": experts, "weights": weights}
    if op == "route_bwd":
        return ctx.route_bwd(s["dweights"], s["x"], s["experts"], score=s["score"], renormalize=s["renorm"])
    if op == "dispatch":
        offsets, position = ctx.expert_order(s["experts"], s["E"])
        return {"rows": ctx.dispatch(s["x"], position, offsets), "offsets": offsets, "position": position}
    if op == "combine":
        return ctx.combine(s["y"], s["position"], s["weights"], s["res"])
    if op == "combine_bwd":
        dy, dweights = ctx.combine_bwd(s["dout"], s["y"], s["position"], s["weights"], s["offsets"])
        return {"dy": dy, "dweights": dweights}
    if op == "linear":
        return ctx.quant_e2m1_gemm(s["x"], s["w"], s["w_tiles"], s["w_row"], s["w_bias"], block=s["block"])
    return ctx.quant_e2m1_gemm_grouped(s["x"], s["offsets"], s["w"], s["w_tiles"], s["w_row"], s["w_bias"], block=s["block"],
                                       position=s["position"])


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------
def work(case):
    op, size = case["op"], 2 if case["dtype"] == "bf16" else 4
    if op == "route":
        T, E, k = case["T"], case["E"], case["k"]
        return {"bytes": size * T * E + 8 * T * k + (4 * E if case["bias"] else 0), "flops": 8 * T * E}
    if op == "route_bwd":
        T, E, k = case["T"], case["E"], case["k"]
        # without renormalised weights every logit of a softmax has a gradient; else the chosen ones' matter
        read = E if case["score"] == "softmax" and not case["renorm"] else k
        return {"bytes": size * T * (read + E) + 8 * T * k, "flops": 8 * T * read}
    if op in ("dispatch", "combine", "combine_bwd"):
        T, cols, k = case["T"], case["cols"], case["k"]
        live = T - case["padded"]
        if op == "dispatch":
            return {"bytes": size * cols * (live + T * k) + 8 * T * k + 4 * case["E"] + 4, "flops": 0}
        if op == "combine":
            return {"bytes": size * cols * (live * k + T * (2 if case["residual"] else 1)) + 8 * T * k, "flops": 2 * live * k * cols}
        return {"bytes": size * cols * (live + live * k + T * k) + 12 * T * k, "flops": 3 * live * k * cols}
    N, K, block, E = case["N"], case["K"], case["block"], case.get("E", 1)
    tokens = case["rows"] if op == "linear" else case["T"]
    rows = tokens * case.get("k", 1)
    used = min(rows, E)     # at most so many experts have rows
    weight = N * ((K + 1) // 2 + -(-K // block)) + N * ((4 if block == 16 else 0) + (4 if case["bias"] else 0))
    plan = 4 * rows + 4 * E if op == "experts" else 0
    return {"bytes": size * (tokens * K + rows * N) + used * weight + plan, "flops": 2 * rows * N * K}


# ---- 64 bits ------------------------------------------------------------------------------------------------------------------
def _scores64(case, x):
    if case["score"] == "sigmoid":
        return 1 / (1 + torch.exp(-x))
    shift = x.max(1, keepdim=True).values
    shift = torch.where(torch.isinf(shift), torch.zeros_like(shift), shift)
    e = torch.exp(x - shift)
    total = e.sum(1, keepdim=True)
    return torch.where(total > 0, e / torch.where(total > 0, total, torch.ones_like(total)), torch.zeros_like(e))


def _exact_route(case, s):
    x = s["x"].double()
    T, E = x.shape
    p = _scores64(case, x)
    c = p.clone()
    if s["balance"] is not None:
        c += s["balance"].double()
    elif case["groups"] == 1:
        c = x.clone()
    c[torch.isinf(x)] = -math.inf
    G = case["groups"]
    if G > 1:
        # one group after the other is taken: the first of the largest sums of the best two
        parts = c.view(T, G, E // G)
        first = parts.max(2)
        rest = parts.scatter(2, first.indices[:, :, None], -math.inf).max(2).values if E // G > 1 else torch.full_like(first.values, -math.inf)
        value = first.values + torch.where(torch.isinf(rest), torch.zeros_like(rest), rest)
        lost = torch.ones_like(value, dtype=torch.bool)
        for _ in range(case["top_groups"]):
            at = (value == value.max(1, keepdim=True).values).to(torch.uint8).argmax(1, keepdim=True)
            lost.scatter_(1, at, False)
            value.scatter_(1, at, -math.inf)
        c = torch.where(lost[:, :, None], torch.full_like(parts, -math.inf), parts).reshape(T, E)
    experts, weights = [], []
    for _ in range(case["k"]):
        top = c.max(1, keepdim=True).values
        at = (c == top).to(torch.uint8).argmax(1, keepdim=True)
        none = torch.isinf(top)
        experts.append(torch.where(none, torch.full_like(at, -1), at))
        weights.append(torch.where(none, torch.zeros_like(top), p.gather(1, at)))
        c.scatter_(1, at, -math.inf)
    experts, weights = torch.cat(experts, 1), torch.cat(weights, 1)
    if case["renorm"]:
        total = weights.sum(1, keepdim=True)
        weights = torch.where(total > 0, weights / total, weights)
    return {"experts": experts.to(torch.int32), "weights": weights}


def _exact_route_bwd(case, s):
    # the Jacobian of the chosen scores, one chosen expert after the other
    x, dw = s["x"].double(), s["dweights"].double()
    p = _scores64(case, x)
    there = s["experts"] >= 0
    at = s["experts"].long().clamp_min(0)
    mine = torch.where(there, p.gather(1, at), torch.zeros_like(dw))
    if case["renorm"]:
        total = mine.sum(1, keepdim=True)
        safe = torch.where(total > 0, total, torch.ones_like(total))
        share = mine / safe
        dp = torch.where(there, dw, torch.zeros_like(dw))
        dp = (dp - torch.einsum("tk,tk->t", dp, share)[:, None]) / safe
    else:
        dp = dw
    dp = torch.where(there, dp, torch.zeros_like(dp))
    dx = torch.zeros_like(x)
    for j in range(case["k"]):
        if case["score"] == "sigmoid":
            dx.scatter_add_(1, at[:, j:j + 1], (dp * mine * (1 - mine))[:, j:j + 1])
        else:
            dx.scatter_add_(1, at[:, j:j + 1], (dp * mine)[:, j:j + 1])
            dx -= (dp * mine)[:, j:j + 1] * p
    return dx


def _rounded64(v):
    """e2m1 by the borders between its numbers: a border goes to the neighbour with the even code."""
    a, out = v.abs(), torch.zeros_like(v)
    for border, up, level in ((0.25, False, 0.5), (0.75, True, 1.0), (1.25, False, 1.5), (1.75, True, 2.0), (2.5, False, 3.0),
                              (3.5, True, 4.0), (5.0, False, 6.0)):
        out = torch.where(a >= border if up else a > border, torch.full_like(out, level), out)
    return out * torch.sign(v)


def _values64(x, block):
    """The values that a row's 4-bit numbers and scales stand for.  Where the definition says binary32, a result in 64 bits is
    rounded to it (of a quotient or a product of two binary32 numbers that is the same number)."""
    rows, cols = x.shape
    f32 = lambda v: v.float().double()
    full = torch.zeros(rows, -(-cols // block) * block, dtype=torch.float64, device=x.device)
    full[:, :cols] = x.double()
    b = full.unflatten(1, (-1, block))
    top = b.abs().max(2, keepdim=True).values
    if block == 32:
        # the exponent field of the binary32 number
        s = torch.exp2(((top.float().view(torch.int32) >> 23) - 129).clamp_min(-127).double())
        return (_rounded64(b / s) * s).flatten(1)[:, :cols]
    g = f32(top.max(1, keepdim=True).values / 2688)
    s = torch.where(g > 0, f32(top / f32(6 * torch.where(g > 0, g, torch.ones_like(g)))), torch.zeros_like(top))
    s = s.float().to(torch.float8_e4m3fn).double()
    unit = f32(s * g)
    r = torch.where(s > 0, f32(1 / torch.where(s > 0, unit, torch.ones_like(unit))), torch.zeros_like(unit))
    return (_rounded64(f32(b * r)) * s * g).flatten(1)[:, :cols]


def _weight64(s, e, block, K):
    codes = s["w"] if s["w"].dim() == 2 else s["w"][e]
    scale = s["w_scale"] if s["w_scale"].dim() == 2 else s["w_scale"][e]
    low, high = codes.to(torch.int32) % 16, codes.to(torch.int32) // 16
    index = torch.empty(codes.shape[0], 2 * codes.shape[1], dtype=torch.int32, device=codes.device)
    index[:, 0::2], index[:, 1::2] = low, high
    magnitude = index[:, :K] % 8
    # exponent and mantissa of e2m1: m / 2 below 1, else (1 + m / 2) 2^(e - 1)
    e2, m1 = (magnitude // 2).double(), (magnitude % 2).double()
    value = torch.where(e2 == 0, 0.5 * m1, (1 + 0.5 * m1) * torch.exp2(e2 - 1)) * (1.0 - 2.0 * (index[:, :K] // 8).double())
    if block == 16:
        row = s["w_row"] if s["w_row"].dim() == 1 else s["w_row"][e]
        unit = scale.view(torch.float8_e4m3fn).double() * row.double()[:, None]
    else:
        unit = torch.exp2(scale.double() - 127)
    at = torch.arange(K, device=codes.device) // block
    return value * unit[:, at]


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "route":
        return _exact_route(case, s)
    if op == "route_bwd":
        return _exact_route_bwd(case, s)
    if op == "dispatch":
        # copies of tokens, and whole numbers: sorted by (expert, token), those without an expert last
        T, k, E = case["T"], case["k"], case["E"]
        expert = s["experts"].flatten().long()
        rank = torch.argsort(torch.where(expert < 0, E, expert) * (T * k) + torch.arange(T * k, device="cuda"))
        live = int((expert >= 0).sum())
        rows = torch.zeros(T * k, case["cols"], dtype=torch.float64, device="cuda")
        rows[:live] = s["x"].double()[rank[:live] // k]
        position = torch.full((T * k,), -1, dtype=torch.int32, device="cuda")
        position[rank[:live]] = torch.arange(live, dtype=torch.int32, device="cuda")
        offsets = (expert[None, :] < torch.arange(E + 1, device="cuda")[:, None]).sum(1) - (T * k - live) if T * k * E < 1 << 28 else \
            torch.searchsorted(expert.sort().values[T * k - live:].contiguous(), torch.arange(E + 1, device="cuda"))
        return {"rows": rows, "offsets": offsets.to(torch.int32), "position": position.view(T, k)}
    if op in ("combine", "combine_bwd"):
        y, position, w = s["y"].double(), s["position"].long(), s["weights"].double()
        if op == "combine":
            out = torch.zeros(case["T"], case["cols"], dtype=torch.float64, device="cuda") if s["res"] is None else s["res"].double()
            for j in range(case["k"]):
                t = (position[:, j] >= 0).nonzero()[:, 0]
                out[t] += w[t, j, None] * y[position[t, j]]
            return out
        dout, dy, dw = s["dout"].double(), torch.zeros_like(y), torch.zeros_like(w)
        for j in range(case["k"]):
            t = (position[:, j] >= 0).nonzero()[:, 0]
            dy[position[t, j]] = w[t, j, None] * dout[t]
            dw[t, j] = torch.einsum("tc,tc->t", y[position[t, j]], dout[t])
        return {"dy": dy, "dweights": dw}
    x, K, block = s["x"], case["K"], case["block"]
    v = _values64(x, block)
    if op == "linear":
        z = torch.einsum("tk,nk->tn", v, _weight64(s, 0, block, K))
        return z if s["w_bias"] is None else z + s["w_bias"].double()
    z = torch.zeros(case["T"] * case["k"], case["N"], dtype=torch.float64, device="cuda")
    for e in range(case["E"]):
        t, j = (s["experts"] == e).nonzero(as_tuple=True)
        if t.numel():
            z[s["position"][t, j].long()] = torch.einsum("tk,nk->tn", v[t], _weight64(s, e, block, K)) + \
                (s["w_bias"][e].double() if s["w_bias"] is not None else 0.0)
    return z
