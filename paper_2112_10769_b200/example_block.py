"""A pre-norm feed-forward block: trained with the 4-bit layers, then answering in 8 bits.

    python -m paper_2112_10769_b200.example_block [--width 512] [--tokens 2048] [--steps 60]

Training: layer norm -> 4-bit linear -> ReLU -> 4-bit linear, added to its input, fitted to a fixed random block
(synthetic regression; the paper's products run in all three directions, the norm's forward and backward pass between
them).  Answering: the same block from int8 weights with a scale per output channel - norm, token quantizer and
product of a layer in one call - for a whole prompt and for one token at a time, and as one of several experts.
"""
from __future__ import annotations

import argparse

import torch

from . import autograd
from .int8 import Int8Experts, Int8Linear


class Block(torch.nn.Module):
    """x + W2 relu(W1 norm(x)) with 4-bit training products."""

    def __init__(self, width: int, hidden: int, device):
        super().__init__()
        self.norm = autograd.LayerNorm(width, device=device)
        self.up = autograd.LuqLinear(width, hidden, n_samples=2, seed=1, device=device)
        self.down = autograd.LuqLinear(hidden, width, n_samples=2, seed=1 << 20, device=device)

    def forward(self, x):
        return x + self.down(torch.relu(self.up(self.norm(x))))

    def exact(self, x):
        """The same block in 32 bits with the trained weights."""
        h = torch.nn.functional.layer_norm(x, (x.shape[-1],), self.norm.weight, self.norm.bias, self.norm.eps)
        return x + torch.relu(h @ self.up.weight.t()) @ self.down.weight.t()


class Int8Block(torch.nn.Module):
    """The trained block in 8 bits."""

    def __init__(self, block: Block):
        super().__init__()
        self.up = Int8Linear.of(block.up, norm=block.norm)
        self.down = Int8Linear.of(block.down)

    def forward(self, x):
        return x + self.down(torch.relu(self.up(x)))


def main(width: int = 512, tokens: int = 2048, steps: int = 60, experts: int = 4, verbose: bool = True):
    device = torch.device("cuda")
    gen = torch.Generator(device).manual_seed(0)
    hidden = 2 * width
    target = [torch.randn(n, k, device=device, generator=gen) * k ** -0.5 for n, k in ((hidden, width), (width, hidden))]

    def batch():
        x = torch.randn(tokens, width, device=device, generator=gen)
        h = torch.relu(torch.nn.functional.layer_norm(x, (width,)) @ target[0].t())
        return x, x + h @ target[1].t()

    torch.manual_seed(0)
    block = Block(width, hidden, device)
    optimizer = torch.optim.Adam(block.parameters(), lr=2e-3)
    losses = []
    for _ in range(steps):
        x, y = batch()
        loss = torch.nn.functional.mse_loss(block(x), y)
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.item())

    with torch.no_grad():
        answer = Int8Block(block)
        x, _ = batch()
        want = block.exact(x)
        prompt = answer(x)
        one_by_one = torch.cat([answer(x[i:i + 1]) for i in range(8)])
        error = ((prompt - want).norm() / (want - x).norm()).item()
        # the block's first product as one of several experts: rows are sent to experts and come back in their order
        weights = torch.stack([block.up.weight] + [torch.randn_like(block.up.weight) * width ** -0.5 for _ in range(experts - 1)])
        layer = Int8Experts(weights)
        expert = torch.randint(experts, (tokens,), device=device, generator=gen)
        routed = layer.route(x, expert)
        ref = torch.einsum("tk,tnk->tn", x[:64], weights[expert[:64]])
        expert_error = ((routed[:64] - ref).norm() / ref.norm()).item()
    result = {"first_loss": losses[0], "last_loss": losses[-1], "int8_error": error, "expert_error": expert_error,
              "one_token_equals_prompt": bool(torch.equal(one_by_one, prompt[:8])),
              "status": autograd.context(device).status()}
    if verbose:
        for k, v in result.items():
            print(f"{k}: {v}")
    return result


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=60)
    a = ap.parse_args()
    main(a.width, a.tokens, a.steps)
