"""Results whose rows lie at 16-byte boundaries but do not end at one: the bytes between belong to the caller.  (Tiled stores write whole
16-byte pieces.)"""
import pytest
import torch

from paper_2608_06812_b200 import binding as ozk
from paper_2608_06812_b200 import lowbit
from tests import test_gpu_fp8_gemm as base
from tests.test_gpu_fp8_pairs import operands, plan

pytestmark = pytest.mark.gpu

# pairs of CTAs with whole sums, over several ranges, with a split K (FP32 scales), and clusters
CASES = [("forward", 2310, 2401, 300, False, (1, 1)), ("wgrad", 2310, 2401, 9000, False, (1, 1)), ("forward", 2310, 2401, 300, True, (1, 1)), ("forward", 300, 601, 9000, True, (1, 9)),
         ("forward", 37, 201, 300, False, (0, 1)), ("forward", 37, 201, 300, True, (0, 1)), ("dgrad", 300, 521, 700, False, (0, 2))]


@pytest.mark.parametrize("way,m,n,k,floats,route", CASES)
@pytest.mark.parametrize("dtype,add", [(torch.bfloat16, False), (torch.float32, False), (torch.float32, True)])
@pytest.mark.parametrize("more", [0, 1, 2, 3, 6])
def test_what_lies_right_of_the_last_column_stays(way, m, n, k, floats, route, dtype, add, more):
    n += more
    piece = 8 if dtype == torch.bfloat16 else 4
    a, b, over = operands(way, m, n, k, more, floats)
    q = plan(a, b, over, dtype)
    assert (q.pairs, q.splits) == route
    whole = torch.full((m + 2, -(-n // piece) * piece), -7.0, dtype=dtype, device="cuda")
    out = whole[1:1 + m, :n]
    before = out.double().cpu().numpy() if add else None
    base.check(lowbit.matmul(a, b, out=out, over_rows=over, accumulate=add), a, b, over, before)
    out.fill_(-7.0)
    assert (whole == -7.0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_neighbouring_columns_of_one_buffer(dtype):
    """Two results side by side in one buffer, the first ending within 16 bytes of the second's start."""
    m, k = 2310, 300
    whole = torch.zeros(m, 4808, dtype=dtype, device="cuda")
    a, b, over = operands("forward", m, 2401, k, 1)
    c, d, _ = operands("forward", m, 2399, k, 2)
    left, right = whole[:, :2401], whole[:, 2401:4800]
    lowbit.matmul(c, d, out=right)
    lowbit.matmul(a, b, out=left)
    base.check(left, a, b, over)
    base.check(right, c, d, over)
    assert (whole[:, 4800:] == 0).all()
