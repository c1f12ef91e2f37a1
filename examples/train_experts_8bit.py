"""Trains a layer of experts behind a norm with 8-bit products and 8-bit AdamW states, then answers tokens with its 8-bit weights.

    python examples/train_experts_8bit.py [steps]

A residual block: the RMS norm of the stream feeds a projection, a router sends each token to two of the experts, rows are put in the
order of the experts, multiplied by the weights of theirs and added up again.  Products, norms and their gradients run in 8 bits; the same network
is trained beside it in 32 bits, on the same data, for comparison.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_06812_b200 import lowbit  # noqa: E402

TOKENS, WIDTH, HIDDEN, EXPERTS, TOP = 1024, 256, 512, 8, 2
EPS = 1e-6


def parameters(seed: int) -> dict[str, torch.Tensor]:
    g = torch.Generator(device="cuda").manual_seed(seed)
    make = lambda *shape: torch.randn(*shape, generator=g, device="cuda") / shape[-1] ** 0.5  # noqa: E731
    return dict(norm=torch.ones(WIDTH, device="cuda"), project=make(WIDTH, WIDTH), router=make(EXPERTS, WIDTH), up=make(EXPERTS, HIDDEN, WIDTH), down=make(EXPERTS, WIDTH, HIDDEN))


def route(h: torch.Tensor, router: torch.Tensor):
    """Each token's experts and gates, as rows in the order of the experts: (token of each row, offsets of the experts, gate of each row)."""
    gates, chosen = torch.topk(torch.softmax(h @ router.T, -1), TOP)
    order = torch.argsort(chosen.reshape(-1), stable=True)
    counts = torch.bincount(chosen.reshape(-1), minlength=EXPERTS)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).int()
    return order // TOP, offsets, gates.reshape(-1)[order]


def plain_norm_linear(x, norm, w, residual=None):
    total = x if residual is None else x + residual
    return torch.nn.functional.linear(total / (total.square().mean(-1, keepdim=True) + EPS).sqrt() * norm, w), total


def plain_expert_linear(x, w, offsets):
    expert = torch.searchsorted(offsets[1:], torch.arange(x.shape[0], device=x.device, dtype=torch.int32), right=True)
    return torch.einsum("ti,toi->to", x, w[expert])


def network(p, x, stream, norm_linear, expert_linear):
    h, total = norm_linear(x, p["norm"], p["project"], stream)
    token, offsets, gates = route(h, p["router"])
    rows = expert_linear(torch.relu(expert_linear(h[token], p["up"], offsets)), p["down"], offsets)
    return total.index_add(0, token, rows * gates[:, None])


def batches(steps: int, seed: int):
    """Inputs and what a fixed network of the same shape answers to them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    teacher = parameters(seed + 1)
    for _ in range(steps):
        x, stream = (torch.randn(TOKENS, WIDTH, generator=g, device="cuda") for _ in range(2))
        yield x, stream, network(teacher, x, stream, plain_norm_linear, plain_expert_linear)


def train(steps: int, bits: int, norm_linear, expert_linear):
    """Losses and parameters of `steps` steps."""
    p = {name: t.requires_grad_() for name, t in parameters(1).items()}
    params = list(p.values())
    grads = [torch.zeros_like(t) for t in params]
    table = lowbit.AdamWTable.zeros(params, grads, bits=bits)
    losses = []
    for step, (x, stream, want) in enumerate(batches(steps, 2), 1):
        loss = (network(p, x, stream, norm_linear, expert_linear) - want).square().mean()
        for g, new in zip(grads, torch.autograd.grad(loss, params)):
            g.copy_(new)
        table.step(lr=1e-3, step=step, betas=(0.9, 0.95), weight_decay=0.01, seed=step if bits == 8 else None)
        losses.append(loss.detach())
    return torch.stack(losses).tolist(), {name: t.detach() for name, t in p.items()}


def answer(p: dict, layers: dict, x: torch.Tensor, stream: torch.Tensor) -> torch.Tensor:
    """The network on tokens in bfloat16, with weights that stay in 8 bits and the stream updated in place."""
    h8 = lowbit.rms_norm(x, p["norm"], stream, eps=EPS, total=stream).rows
    h = lowbit.matmul(h8, layers["project"])
    token, offsets, gates = route(h.float(), p["router"])
    hidden = torch.relu(lowbit.grouped_matmul(lowbit.quantize_lines(h[token])[0], layers["up"], offsets))
    rows = lowbit.grouped_matmul(lowbit.quantize_lines(hidden)[0], layers["down"], offsets)
    return stream.float().index_add(0, token, rows.float() * gates[:, None])


def main(steps: int = 200) -> tuple[list[float], list[float], float]:
    plain, _ = train(steps, 32, plain_norm_linear, plain_expert_linear)
    eight, p = train(steps, 8, lambda *a: lowbit.norm_linear(*a, eps=EPS), lowbit.expert_linear)
    for step in sorted({0, steps // 10, steps // 3, steps - 1}):
        print(f"step {step + 1:4d}   loss in 32 bits {plain[step]:.5f}   in 8 bits {eight[step]:.5f}")
    layers = dict(project=lowbit.quantize_tiles(p["project"]), up=lowbit.quantize_experts(p["up"]), down=lowbit.quantize_experts(p["down"]))
    x, stream, _ = next(batches(1, 3))
    x, stream = x.bfloat16()[:64], stream.bfloat16()[:64]
    together = answer(p, layers, x, stream.clone())
    alone = torch.cat([answer(p, layers, x[i:i + 1], stream[i:i + 1].clone()) for i in range(64)])
    off = float((together - alone).norm() / together.norm())
    lowbit.check_async()
    print(f"64 tokens answered one by one and together differ by {off:.1e} of their norm")
    return plain, eight, off


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 200)
