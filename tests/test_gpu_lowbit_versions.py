"""Writes of the 8-bit operators to tensors that autograd has saved: the backward pass raises, as after torch's own in-place operations."""
import pytest
import torch

from paper_2608_06812_b200 import lowbit

pytestmark = pytest.mark.gpu

CHANGED = "modified by an inplace operation"


def saved(t):
    """The loss of a product that keeps t for the gradient of its other factor."""
    other = torch.ones_like(t, requires_grad=True)
    return (other * t.detach() if not t.requires_grad else other * t).float().sum()


def test_results_written_over():
    x = torch.randn(40, 256, device="cuda")
    a, b, out = lowbit.quantize_lines(x)[0], lowbit.quantize_tiles(x), torch.zeros(40, 40, device="cuda")
    loss = saved(out)
    lowbit.matmul(a, b, out=out)
    with pytest.raises(RuntimeError, match=CHANGED):
        loss.backward()
    saved(out).backward()


def test_a_step_between_forward_and_backward():
    for bits in (8, 32):
        p, copy = torch.randn(300, device="cuda", requires_grad=True), torch.zeros(300, dtype=torch.bfloat16, device="cuda")
        table = lowbit.AdamWTable.zeros([p], [torch.ones(300, device="cuda")], bits=bits, copies=[copy])
        for t in (p, copy):
            loss = saved(t)
            table.step(lr=1e-3, step=1)
            with pytest.raises(RuntimeError, match=CHANGED):
                loss.backward()
            saved(t).backward()


def test_quantised_again():
    x = torch.randn(40, 256, device="cuda")
    r, c, t = lowbit.Fp8Matrix.empty(40, 256, "rows"), lowbit.Fp8Matrix.empty(40, 256, "cols"), lowbit.Fp8Matrix.empty(40, 256, "tiles")
    versions = lambda: [(m.codes._version, m.scales._version) for m in (r, c, t)]  # noqa: E731
    before = versions()
    lowbit.quantize_lines(x, r, c)
    lowbit.quantize_tiles(x, t)
    assert all(n > o for a, b in zip(before, versions()) for o, n in zip(a, b))


def test_tensors_of_inference_mode_have_no_versions():
    with torch.inference_mode():
        x = torch.randn(40, 256, device="cuda")
        a, b, out = lowbit.Fp8Matrix.empty(40, 256, "rows"), lowbit.Fp8Matrix.empty(40, 256, "tiles"), torch.zeros(40, 40, device="cuda")
        lowbit.quantize_lines(x, a)
        lowbit.quantize_tiles(x, b)
        lowbit.matmul(a, b, out=out)
        p = [torch.zeros(300, device="cuda")]
        lowbit.AdamWTable.zeros(p, [torch.ones(300, device="cuda")], copies=[torch.zeros(300, dtype=torch.bfloat16, device="cuda")]).step(lr=1e-3, step=1)
        assert (p[0] != 0).all()
    assert torch.equal(out, lowbit.matmul(a, b, dtype=torch.float32))
