"""A layer of experts: trained with the 4-bit layers, then answering in microscaled 4-bit floating point and in 8 bits.

    python -m paper_2112_10769_b200.example_experts [--width 256] [--tokens 2048] [--experts 8] [--steps 40]

Training: layer norm -> router (sigmoid scores, bias for balance, two of the experts for each token) -> the tokens' copies in the
experts' order -> every expert's two 4-bit linear layers -> their weighted sum, added to the layer's input; fitted to a fixed random
layer (synthetic regression).  Gradients run through the sum, the copies and the router's scores.  Answering: the same layer from
e2m1 weights with a scale for each block (the first product takes the tokens and the copies' positions), or from int8 ones.
"""
from __future__ import annotations

import argparse

import torch

from . import autograd, experts
from .e2m1 import E2m1Experts
from .int8 import Int8Experts


class ExpertLayer(torch.nn.Module):
    """x + sum of w_j W2_e relu(W1_e norm(x)) over a token's experts e, with 4-bit training products."""

    def __init__(self, width: int, hidden: int, n_experts: int, k: int, device):
        super().__init__()
        self.norm = autograd.LayerNorm(width, device=device)
        self.router = experts.Router(width, n_experts, k, score="sigmoid", balance=True, device=device)
        self.up = torch.nn.ModuleList(autograd.LuqLinear(width, hidden, n_samples=2, seed=1 + 1000 * e, device=device) for e in range(n_experts))
        self.down = torch.nn.ModuleList(autograd.LuqLinear(hidden, width, n_samples=2, seed=(1 << 20) + 1000 * e, device=device)
                                        for e in range(n_experts))

    def forward(self, x):
        h = self.norm(x)
        chosen, weights = self.router(h)
        self.offsets, position = experts.order(chosen, len(self.up))
        rows = experts.dispatch(h, position, self.offsets)
        ends = self.offsets.tolist()                   # (the 4-bit training products take their sizes from the host)
        y = [self.down[e](torch.relu(self.up[e](rows[a:b]))) for e, (a, b) in enumerate(zip(ends, ends[1:])) if b > a]
        y = torch.cat([*y, rows[ends[-1]:]])
        return experts.combine(y, position, weights, self.offsets, residual=x)


class ExpertAnswer(torch.nn.Module):
    """The trained layer answering; nothing waits for the device.  ``block``: of e2m1's scales, or None: int8."""

    def __init__(self, layer: ExpertLayer, block: int | None = 16):
        super().__init__()
        self.norm, self.router, self.n_experts = layer.norm, layer.router, len(layer.up)
        up, down = (torch.stack([m.weight.detach() for m in part]) for part in (layer.up, layer.down))
        self.up, self.down = (Int8Experts(w) if block is None else E2m1Experts(w, block=block) for w in (up, down))

    @torch.no_grad()
    def forward(self, x):
        h = self.norm(x)
        chosen, weights = self.router(h)
        offsets, position = experts.order(chosen, self.n_experts)
        if isinstance(self.up, E2m1Experts):
            y = self.up(h, offsets, position)
        else:
            y = self.up(experts.dispatch(h, position, offsets), offsets)
        y = self.down(torch.relu(y), offsets)
        return experts.combine(y, position, weights, offsets, residual=x)


def exact(layer: ExpertLayer, x):
    """The same layer in 32 bits with the trained weights, every token through all experts."""
    h = torch.nn.functional.layer_norm(x, (x.shape[-1],), layer.norm.weight, layer.norm.bias, layer.norm.eps)
    chosen, weights = layer.router(h)
    out = x.clone()
    for e in range(len(layer.up)):
        w = torch.where(chosen == e, weights, torch.zeros_like(weights)).sum(1, keepdim=True)
        out += w * (torch.relu(h @ layer.up[e].weight.t()) @ layer.down[e].weight.t())
    return out


def main(width: int = 256, tokens: int = 2048, n_experts: int = 8, k: int = 2, steps: int = 40, verbose: bool = True):
    device = torch.device("cuda")
    gen = torch.Generator(device).manual_seed(0)
    torch.manual_seed(0)
    target = ExpertLayer(width, 2 * width, n_experts, k, device)
    layer = ExpertLayer(width, 2 * width, n_experts, k, device)
    optimizer = torch.optim.Adam(layer.parameters(), lr=2e-3)
    losses = []
    for _ in range(steps):
        x = torch.randn(tokens, width, device=device, generator=gen)
        with torch.no_grad():
            y = exact(target, x)
        loss = torch.nn.functional.mse_loss(layer(x), y)
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        layer.router.rebalance(layer.offsets)
        losses.append(loss.item())
    x = torch.randn(tokens, width, device=device, generator=gen)
    with torch.no_grad():
        want = exact(layer, x)
    result = {"first_loss": losses[0], "last_loss": losses[-1]}
    for name, block in (("e2m1_block16", 16), ("e2m1_block32", 32), ("int8", None)):
        got = ExpertAnswer(layer, block)(x)
        result[name + "_error"] = ((got - want).norm() / (want - x).norm()).item()
    result["status"] = autograd.context(device).status()
    if verbose:
        for name, value in result.items():
            print(f"{name}: {value}")
    return result


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--experts", type=int, default=8)
    ap.add_argument("--steps", type=int, default=40)
    a = ap.parse_args()
    main(a.width, a.tokens, a.experts, steps=a.steps)
