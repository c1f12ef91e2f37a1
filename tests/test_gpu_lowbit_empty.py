"""A layer without inputs, without outputs, without tokens."""
import pytest
import torch

from paper_2608_06812_b200 import lowbit

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,inputs,outputs", [((3,), 0, 4), ((2, 3), 0, 4), ((), 0, 4), ((3,), 5, 0), ((2, 0), 5, 4), ((0,), 0, 4), ((), 5, 4)])
def test_linear(tokens, inputs, outputs):
    x, w = torch.ones(*tokens, inputs, device="cuda", requires_grad=True), torch.ones(outputs, inputs, device="cuda", requires_grad=True)
    y = lowbit.linear(x, w)
    want = torch.nn.functional.linear(x, w)
    assert y.shape == want.shape and torch.equal(y, want)
    y.sum().backward()
    dx, dw = x.grad, w.grad
    x.grad = w.grad = None
    want.sum().backward()
    assert dx.shape == x.shape and torch.equal(dx, x.grad) and torch.equal(dw, w.grad)
