"""Trains a two-layer perceptron with 8-bit products and 8-bit AdamW states, then answers single tokens with its 8-bit weights.

    python examples/train_8bit.py [steps]

Every step quantises activations, weights and output gradients to E4M3 with a scale for each block of 128, forms the forward
products and both gradients on the tensor cores, and updates all tensors in one AdamW launch.  The same
network is trained beside it in 32 bits, on the same data, for comparison.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_06812_b200 import lowbit  # noqa: E402

TOKENS, INPUTS, HIDDEN, OUTPUTS = 2048, 512, 1024, 384


def batches(steps: int, seed: int):
    """Inputs and what a fixed network of the same shape answers to them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    teacher = [torch.randn(HIDDEN, INPUTS, generator=g, device="cuda") / INPUTS ** 0.5, torch.randn(OUTPUTS, HIDDEN, generator=g, device="cuda") / HIDDEN ** 0.5]
    for _ in range(steps):
        x = torch.randn(TOKENS, INPUTS, generator=g, device="cuda")
        yield x, torch.relu(x @ teacher[0].T) @ teacher[1].T


def weights(seed: int):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(o, i, generator=g, device="cuda") / i ** 0.5) for o, i in ((HIDDEN, INPUTS), (OUTPUTS, HIDDEN))]


def train(steps: int, bits: int, product) -> tuple[list[float], list[torch.Tensor]]:
    """Losses and weights of `steps` steps with `product` for the layers and states of `bits` bits."""
    params = [w.requires_grad_() for w in weights(1)]
    grads = [torch.zeros_like(p) for p in params]
    table = lowbit.AdamWTable.zeros(params, grads, bits=bits)
    losses = []
    for step, (x, want) in enumerate(batches(steps, 2), 1):
        loss = (product(torch.relu(product(x, params[0])), params[1]) - want).square().mean()
        for g, new in zip(grads, torch.autograd.grad(loss, params)):
            g.copy_(new)
        norm = torch.stack([g.square().sum() for g in grads]).sum().sqrt()
        clip = torch.clamp(1.0 / (norm + 1e-6), max=1.0)
        table.step(lr=2e-3, step=step, betas=(0.9, 0.95), weight_decay=0.01, seed=step if bits == 8 else None, grad_scale=clip)
        losses.append(loss.detach())
    return torch.stack(losses).tolist(), [p.detach() for p in params]


def answer(tokens: torch.Tensor, layers: list[lowbit.Fp8Matrix]) -> torch.Tensor:
    """The network on [n, INPUTS] tokens in bfloat16, with weights that stay in 8 bits."""
    for i, w in enumerate(layers):
        tokens = lowbit.matmul(lowbit.quantize_lines(torch.relu(tokens) if i else tokens)[0], w)
    return tokens


def main(steps: int = 300) -> tuple[list[float], list[float], float]:
    plain, _ = train(steps, 32, torch.nn.functional.linear)
    eight, params = train(steps, 8, lowbit.linear)
    for step in sorted({0, steps // 10, steps // 3, steps - 1}):
        print(f"step {step + 1:4d}   loss in 32 bits {plain[step]:.5f}   in 8 bits {eight[step]:.5f}")
    layers = [lowbit.quantize_tiles(p) for p in params]
    x, _ = next(batches(1, 3))
    x = x.bfloat16()
    together = answer(x[:64], layers)
    alone = torch.cat([answer(x[i:i + 1], layers) for i in range(64)])
    off = float((together.float() - alone.float()).norm() / together.float().norm())
    lowbit.check_async()
    print(f"64 tokens answered one by one and together differ by {off:.1e} of their norm")
    return plain, eight, off


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 300)
