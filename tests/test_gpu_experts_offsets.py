"""Offsets that fall or leave the rows are read as the nearest that do not, also where there is nothing to sum (K = 0): rows of segments become zero, rows of nobody stay."""
import pytest
import torch

from paper_2608_06812_b200 import lowbit

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bad,first,behind", [([0, 100, 50, 400, 10], 0, 300), ([-5, 20, 20, 7, -3], 0, 20), ([250, 0, 0, 260, 10], 250, 260), ([3, 2, 1, 0, 0], 3, 3), ([400, 9, 9, 9, 9], 300, 300),
                                              ([10] + [0] * 70 + [200] + [0] * 950 + [150, 0], 10, 200), ([0] * 1024 + [299], 0, 299)])
def test_falling_offsets_with_nothing_to_sum(bad, first, behind, dtype):
    experts = len(bad) - 1
    a, w, offsets = lowbit.Fp8Matrix.empty(300, 0, lowbit.ROWS), lowbit.Fp8Experts.empty(experts, 40, 0), torch.tensor(bad, dtype=torch.int32, device="cuda")
    out = torch.full((300, 40), -7.0, dtype=dtype, device="cuda")
    lowbit.grouped_matmul(a, w, offsets, out=out)
    want = torch.full_like(out, -7.0)
    want[first:behind] = 0.0
    assert torch.equal(out, want)
    assert (lowbit.grouped_matmul(a, w, offsets, dtype=dtype) == 0).all()


@pytest.mark.parametrize("bad,first,behind", [([0, 100, 50, 400, 10], 0, 300), ([250, 0, 0, 260, 10], 250, 260), ([3, 2, 1, 0, 0], 3, 3)])
def test_the_same_rows_with_something_to_sum(bad, first, behind):
    x = torch.ones(300, 64, device="cuda")
    w = lowbit.quantize_experts(torch.ones(4, 40, 64, device="cuda"))
    out = torch.full((300, 40), -7.0, device="cuda")
    lowbit.grouped_matmul(lowbit.quantize_lines(x)[0], w, torch.tensor(bad, dtype=torch.int32, device="cuda"), out=out)
    want = torch.full_like(out, -7.0)
    want[first:behind] = 64.0
    assert torch.equal(out, want)
    lowbit.check_async()
