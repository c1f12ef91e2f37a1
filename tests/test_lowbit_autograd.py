"""What `lowbit.linear` tells autograd, on the CPU: exact stand-ins take the places of the kernels."""
import pytest
import torch

from paper_2608_06812_b200 import lowbit


class Matrix:
    def __init__(self, x, kind):
        self.codes, self.scales, self.kind, (self.rows, self.cols), self.index = x, torch.zeros(1), kind, x.shape, 0


@pytest.fixture(autouse=True)
def asked(monkeypatch):
    """Replaces the kernels; the list of forms that quantize_lines was asked for."""
    forms = []

    def quantize_lines(x, rows=True, cols=False):
        forms.append((bool(rows), bool(cols)))
        return Matrix(x.detach().clone(), "rows") if rows else None, Matrix(x.detach().clone(), "cols") if cols else None

    def matmul(a, b, out=None, over_rows=False, dtype=torch.bfloat16, accumulate=False):
        A = a.codes.T if a.kind == "cols" else a.codes
        B = b.codes.T if b.kind == "cols" or over_rows else b.codes
        return (A @ B.T).to(dtype)

    monkeypatch.setattr(lowbit, "quantize_lines", quantize_lines)
    monkeypatch.setattr(lowbit, "quantize_tiles", lambda x, out=None: Matrix(x.detach().clone(), "tiles"))
    monkeypatch.setattr(lowbit, "matmul", matmul)
    return forms


def arguments():
    g = torch.Generator().manual_seed(0)
    return torch.randn(5, 6, generator=g, requires_grad=True), torch.randn(4, 6, generator=g, requires_grad=True)


def test_first_derivatives():
    x, w = arguments()
    dx, dw = torch.autograd.grad(lowbit.linear(x, w).square().sum(), (x, w))
    y = torch.nn.functional.linear(x, w)
    ex, ew = torch.autograd.grad(y.square().sum(), (x, w))
    assert torch.allclose(dx, ex) and torch.allclose(dw, ew)


def test_second_derivatives_are_refused():
    """The gradients are formed in 8 bits outside autograd: a penalty on them would be left out without a word."""
    x, w = arguments()
    dx, = torch.autograd.grad(lowbit.linear(x, w).square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        dx.square().sum().backward()


def test_columns_are_quantised_only_for_a_weight_gradient(asked):
    """The form of x by columns serves the weight gradient alone."""
    x, w = arguments()
    lowbit.linear(x, w)
    assert asked.pop() == (True, True)
    for call in (lambda: lowbit.linear(x, w.detach()), lambda: lowbit.linear(x.detach(), w.detach())):
        call()
        assert asked.pop() == (True, False)
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            lowbit.linear(x, w)
            assert asked.pop() == (True, False), mode


def test_kept_weights_that_do_not_fit_are_refused():
    """Weights by rows serve the forward product only: summed over their rows, dx would be dy w^T of a square weight."""
    x, w = arguments()
    square = torch.randn(6, 6, generator=torch.Generator().manual_seed(1), requires_grad=True)
    tiles, rows, cols = (Matrix(square.detach(), k) for k in ("tiles", "rows", "cols"))
    floats = Matrix(square.detach(), "tiles")
    floats.scales = torch.ones(1, 1)
    for m in (tiles, rows, cols):
        m.scales = torch.zeros(1, 1, dtype=torch.uint8)
    for bad in (rows, cols, floats):
        with pytest.raises(ValueError):
            lowbit.linear(x, square, bad)
    for bad in (cols, floats):
        with torch.no_grad(), pytest.raises(ValueError):
            lowbit.linear(x, square, bad)
    with pytest.raises(ValueError):
        lowbit.linear(x, w, tiles)                     # another weight's
    want = torch.nn.functional.linear(x, square)
    assert torch.allclose(lowbit.linear(x, square, tiles), want)
    with torch.no_grad():
        assert torch.allclose(lowbit.linear(x, square, rows), want)
    y = lowbit.linear(x.detach(), square, rows)        # no gradient of x: the weights are summed over their columns only
    assert torch.allclose(torch.autograd.grad(y.sum(), square)[0], torch.autograd.grad(want.sum(), square)[0])


def test_kept_weights_written_again_before_the_backward_pass_are_noticed():
    x, w = arguments()
    w8 = Matrix(w.detach().clone(), "tiles")
    w8.scales = torch.zeros(1, 1, dtype=torch.uint8)
    for part in (w8.codes, w8.scales):
        y = lowbit.linear(x, w, w8)
        part.zero_()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()
    y = lowbit.linear(x.detach(), w, w8)     # the weight gradient does not read them
    w8.codes.zero_()
    y.sum().backward()
    with torch.inference_mode():             # tensors of inference mode have no versions, and serve as before
        w8 = Matrix(w.detach().clone(), "tiles")
        w8.scales = torch.zeros(1, 1, dtype=torch.uint8)
    x.grad = None
    lowbit.linear(x, w, w8).sum().backward()
    assert torch.allclose(x.grad, w.detach().sum(0).expand(5, -1))


def test_a_graph_may_be_walked_again():
    x, w = arguments()
    loss = lowbit.linear(x, w).sum()
    loss.backward()
    first = x.grad.clone()
    loss.backward()
    assert torch.equal(x.grad, 2 * first)
