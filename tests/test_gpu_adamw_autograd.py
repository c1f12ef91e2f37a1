"""An AdamW table over gradients that autograd owns: a gradient that has been replaced is noticed, not stepped from memory of its past."""
import pytest
import torch

from paper_2608_06812_b200 import lowbit

pytestmark = pytest.mark.gpu


def network():
    g = torch.Generator().manual_seed(0)
    params = [torch.nn.Parameter(torch.randn(n, generator=g).cuda()) for n in (300, 5000, 7)]
    x = [torch.randn(p.numel(), generator=g).cuda() for p in params]

    def backward():
        sum((p * a).square().sum() for p, a in zip(params, x)).backward()

    backward()
    return params, backward


@pytest.mark.parametrize("bits", [8, 32])
def test_gradients_that_moved_are_refused(bits):
    params, backward = network()
    table = lowbit.AdamWTable.zeros(params, [p.grad for p in params], bits=bits)
    table.step(lr=1e-2, step=1)
    for p in params:
        p.grad = None                       # zero_grad() by default
    before = [p.detach().clone() for p in params]
    with pytest.raises(RuntimeError, match="gradient"):
        table.step(lr=1e-2, step=2)
    backward()
    kept = params[1].grad
    params[1].grad = torch.zeros_like(kept)  # one of them elsewhere
    with pytest.raises(RuntimeError, match="gradient"):
        table.step(lr=1e-2, step=2)
    assert all(torch.equal(p, b) for p, b in zip(params, before))
    lowbit.AdamWTable(params, [p.grad for p in params], *(table.tensors[k] for k in ("m", "v", "m_scale", "v_scale"))).step(lr=1e-2, step=2)
    assert not torch.equal(params[0], before[0])


def test_gradients_that_stay_are_followed():
    params, backward = network()
    other, _ = network()
    table = lowbit.AdamWTable.zeros(params, [p.grad for p in params], bits=32)
    optimizer = torch.optim.AdamW(other, lr=1e-2, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01)
    for step in range(1, 4):
        for p in params:
            p.grad.zero_()
        backward()
        for p, q in zip(params, other):
            q.grad = p.grad.clone()
        optimizer.step()
        table.step(lr=1e-2, step=step)
    # a step is at most about lr; each of the three differs by the roundings of its moments and quotient, far below 2^-20 of lr
    assert all(((p - q).abs() <= 3 * (1e-2 * 2.0 ** -20 + 2.0 ** -23 * q.abs())).all() for p, q in zip(params, other))


def test_gradients_of_the_callers_own_are_not_watched():
    params, backward = network()
    table = lowbit.AdamWTable.zeros(params, [p.grad.clone() for p in params], bits=32)
    for p in params:
        p.grad = None
    table.step(lr=1e-2, step=1)
    view = [p.detach().clone().requires_grad_() for p in params]
    for v, p in zip(view, params):
        v.grad = torch.ones_like(p)
    table = lowbit.AdamWTable.zeros(view, [v.grad.view(-1) for v in view])   # the same memory by another tensor
    table.step(lr=1e-2, step=1)
    view[0].grad = None
    with pytest.raises(RuntimeError, match="gradient"):
        table.step(lr=1e-2, step=2)


def test_params_without_elements_are_not_watched():
    p, q = torch.nn.Parameter(torch.zeros(0, device="cuda")), torch.nn.Parameter(torch.zeros(5, device="cuda"))
    p.grad = torch.zeros(0, device="cuda")
    table = lowbit.AdamWTable.zeros([p, q], [torch.zeros(0, device="cuda"), torch.ones(5, device="cuda")])
    p.grad = None
    table.step(lr=1e-2, step=1)
    assert (q != 0).all()
