"""The 8-bit operators together: a linear layer's gradients against the formula and against differences, and a network that trains."""
import numpy as np
import pytest
import torch

from paper_2608_06812_b200 import lowbit

pytestmark = pytest.mark.gpu


def integers(shape, most, seed):
    return torch.randint(-most, most + 1, shape, generator=torch.Generator().manual_seed(seed)).float().cuda()


@pytest.mark.parametrize("tokens,inputs,outputs", [(1, 128, 16), (5, 130, 40), (200, 300, 150), (129, 257, 384)])
def test_gradients_are_those_of_the_formula(tokens, inputs, outputs):
    """Whole numbers up to 4 are E4M3 values under any power-of-two scale a block of them gets, and their sums are exact in FP32: the
    8-bit layer is then the exact one, and so are its gradients."""
    x, w, dy = integers((tokens, inputs), 4, 1).requires_grad_(), integers((outputs, inputs), 4, 2).requires_grad_(), integers((tokens, outputs), 4, 3)
    y = lowbit.linear(x, w)
    assert torch.equal(y, (x.double() @ w.double().T).float())
    y.backward(dy)
    assert torch.equal(x.grad, (dy.double() @ w.double()).float())
    assert torch.equal(w.grad, (dy.double().T @ x.double()).float())


def test_gradients_are_those_of_differences():
    """The layer is linear in each argument: central differences by a whole step are its gradient, to the last bit here."""
    x, w, dy = integers((6, 140), 4, 4), integers((20, 140), 4, 5), integers((6, 20), 4, 6)
    xg, wg = x.clone().requires_grad_(), w.clone().requires_grad_()
    (lowbit.linear(xg, wg) * dy).sum().backward()
    f = lambda x, w: float((lowbit.linear(x, w).double() * dy.double()).sum())  # noqa: E731
    rng = np.random.default_rng(0)
    for _ in range(12):
        i, j = int(rng.integers(6)), int(rng.integers(140))
        e = torch.zeros_like(x)
        e[i, j] = 1.0
        assert (f(x + e, w) - f(x - e, w)) / 2 == float(xg.grad[i, j])
        i, j = int(rng.integers(20)), int(rng.integers(140))
        e = torch.zeros_like(w)
        e[i, j] = 1.0
        assert (f(x, w + e) - f(x, w - e)) / 2 == float(wg.grad[i, j])


def test_gradients_of_ordinary_values():
    """Each 8-bit operand is off by at most 2^-4 of an element (half a unit of three fraction bits) or 2^-10 of its block's
    scale unit: independent errors of relative size 2^-4 / sqrt(3) at most in two factors, 5.1 % of the products' norm."""
    g = torch.Generator().manual_seed(0)
    x, w, dy = (torch.randn(s, generator=g).cuda() for s in ((500, 700), (300, 700), (500, 300)))
    xg, wg = x.clone().requires_grad_(), w.clone().requires_grad_()
    y = lowbit.linear(xg, wg)
    y.backward(dy)
    for got, want in ((y, x @ w.T), (xg.grad, dy @ w), (wg.grad, dy.T @ x)):
        assert (got - want).norm() < 0.051 * want.norm()


def test_batched_input_partial_gradients_and_16_bits():
    x, w = torch.randn(2, 3, 64, device="cuda", dtype=torch.bfloat16), torch.randn(32, 64, device="cuda", requires_grad=True)
    y = lowbit.linear(x, w)
    assert y.shape == (2, 3, 32) and y.dtype == torch.bfloat16
    y.float().sum().backward()
    assert w.grad.shape == w.shape and w.grad.dtype == torch.float32
    x.requires_grad_()
    kept = lowbit.quantize_tiles(w.detach())
    y = lowbit.linear(x, w.detach(), kept)
    y.float().sum().backward()
    assert x.grad.shape == x.shape and x.grad.dtype == torch.bfloat16


def test_strided_and_empty_arguments():
    x, w = integers((130, 20), 4, 7).T, integers((130, 40), 4, 8).T      # neither has contiguous rows
    x, w = x.requires_grad_(), w.requires_grad_()
    y = lowbit.linear(x, w)
    y.backward(torch.ones(40, device="cuda").expand(20, 40))
    assert torch.equal(y, (x.double() @ w.double().T).float())
    assert torch.equal(x.grad, w.double().sum(0).float().expand(20, -1)) and torch.equal(w.grad, x.double().sum(0).float().expand(40, -1))
    y = lowbit.linear(x, w)
    x.grad = w.grad = None
    y.sum().backward()                                                     # a gradient expanded from one number
    assert torch.equal(x.grad, w.double().sum(0).float().expand(20, -1))
    x, w = torch.zeros(0, 64, device="cuda", requires_grad=True), torch.randn(32, 64, device="cuda", requires_grad=True)
    y = lowbit.linear(x, w)
    y.sum().backward()
    assert y.shape == (0, 32) and x.grad.shape == (0, 64) and (w.grad == 0).all()


def test_the_example_learns():
    """The 8-bit run follows the 32-bit one: both lose 80 % of the loss, and the 8-bit one ends within a factor of two."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import train_8bit
    plain, eight, off = train_8bit.main(200)
    assert plain[-1] < 0.2 * plain[0] and eight[-1] < 0.2 * eight[0]
    assert eight[-1] < 2.0 * plain[-1]
    assert off < 2e-3
