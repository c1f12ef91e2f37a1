"""The block-scaled product on pairs of CTAs: more tiles than pairs, more than one band of them, remainders, sums over several ranges, added
and strided results; and every combination of operand kinds.  Each test asserts, by the host's plan, that its product goes where it means to.
Bounds: those of the product's other tests."""
import pytest
import torch

from paper_2608_06812_b200 import binding as ozk
from paper_2608_06812_b200 import lowbit
from tests import test_gpu_fp8_gemm as base

pytestmark = pytest.mark.gpu


def operands(way, m, n, k, seed, floats=False):
    if way == "rows x cols":
        return base.random_matrix(m, k, "rows", seed), base.random_matrix(k, n, "cols", seed + 1), False
    if way == "cols x rows":
        return base.random_matrix(k, m, "cols", seed), base.random_matrix(n, k, "rows", seed + 1), False
    if way == "tiles x tiles":
        return base.random_matrix(m, k, "tiles", seed), base.random_matrix(n, k, "tiles", seed + 1), False
    if way == "tiles x tiles over rows":
        return base.random_matrix(m, k, "tiles", seed), base.random_matrix(k, n, "tiles", seed + 1), True
    if way == "tiles x rows":
        return base.random_matrix(m, k, "tiles", seed), base.random_matrix(n, k, "rows", seed + 1), False
    if way == "cols x tiles":
        return base.random_matrix(k, m, "cols", seed), base.random_matrix(k, n, "tiles", seed + 1), True
    return base.operands(way, m, n, k, seed, floats)


def plan(a, b, over, dtype):
    a_over = a.kind == "cols" or (a.kind == "tiles" and b.kind == "cols")
    b_over = b.kind == "cols" or (b.kind == "tiles" and over)
    m, k = (a.cols, a.rows) if a_over else (a.rows, a.cols)
    return ozk.ozk_fp8_gemm_plan(m, b.cols if b_over else b.rows, k, a._operand[a_over], b._operand[b_over], ozk.OZK_BF16 if dtype == torch.bfloat16 else ozk.OZK_F32)


WAYS = ["forward", "dgrad", "wgrad", "lines", "mixed"]
MORE_WAYS = ["rows x cols", "cols x rows", "tiles x tiles", "tiles x tiles over rows", "tiles x rows", "cols x tiles"]
TWO = [torch.bfloat16, torch.float32]
# 100 tiles on 74 pairs (two rounds), 54 tiles in two bands of 16 rows of tiles, 110 tiles of a single short block, 228 tiles in three bands
SIZES = [(2500, 2310, 700), (4400, 600, 1100), (2305, 2561, 96), (9700, 1400, 260)]


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype", TWO)
def test_product(way, m, n, k, dtype):
    a, b, over = operands(way, m, n, k, m + n + k)
    q = plan(a, b, over, dtype)
    assert q.pairs and q.splits == 1 and q.tiles == -(-m // 256) * -(-n // 256)
    base.check(lowbit.matmul(a, b, over_rows=over, dtype=dtype), a, b, over)
    lowbit.check_async()


@pytest.mark.parametrize("way", MORE_WAYS)
@pytest.mark.parametrize("m,n,k,pairs", [(5, 300, 500, 0), (33, 200, 129, 0), (300, 520, 700, 0), (2305, 2561, 300, 1)])
@pytest.mark.parametrize("dtype", TWO)
def test_every_combination_of_kinds(way, m, n, k, pairs, dtype):
    a, b, over = operands(way, m, n, k, m + n + k)
    assert plan(a, b, over, dtype).pairs == pairs
    base.check(lowbit.matmul(a, b, over_rows=over, dtype=dtype), a, b, over)
    lowbit.check_async()


@pytest.mark.parametrize("m,n,k", [*SIZES, (700, 2600, 1300)])
@pytest.mark.parametrize("dtype", TWO)
def test_float_scales(m, n, k, dtype):
    a, b, over = operands("forward", m, n, k, m + n + k, floats=True)
    q = plan(a, b, over, dtype)
    assert q.pairs and q.splits == 1
    base.check(lowbit.matmul(a, b, dtype=dtype), a, b, over)
    lowbit.check_async()


@pytest.mark.parametrize("way,floats", [("wgrad", False), ("forward", False), ("forward", True)])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("m,n,k", [(2310, 2500, 9000), (300, 301, 40000), (2500, 2310, 700), (300, 600, 9000)])
def test_ranges_splits_and_sums(way, floats, add, m, n, k):
    """FP32 results: several ranges of a tile added in order, partial sums of a split K, and both onto what is there."""
    a, b, over = operands(way, m, n, k, m + n + k, floats)
    q = plan(a, b, over, torch.float32)
    if (m, n, k) != (300, 600, 9000) or floats:
        assert q.pairs and (q.splits > 1) == (m == 300)
    c = torch.randn(m, n, generator=torch.Generator().manual_seed(1)).mul(float(k) ** 0.5).cuda()
    before = c.double().cpu().numpy() if add else None
    base.check(lowbit.matmul(a, b, out=c, over_rows=over, accumulate=add), a, b, over, before)
    lowbit.check_async()


@pytest.mark.parametrize("floats", [False, True])
@pytest.mark.parametrize("dtype,add", [(torch.bfloat16, False), (torch.float32, False), (torch.float32, True)])
@pytest.mark.parametrize("pad", [1, 4, 8])
def test_strided_results_leave_their_surroundings(floats, dtype, add, pad):
    """Rows that are not multiples of 16 bytes are stored element by element, others by whole boxes."""
    m, n, k = 2310, 2401, 300
    a, b, over = operands("forward", m, n, k, pad, floats)
    assert plan(a, b, over, dtype).pairs
    whole = torch.full((m + 2, n + 2 * pad), -7.0, dtype=dtype, device="cuda")
    out = whole[1:1 + m, pad:pad + n]
    before = out.double().cpu().numpy() if add else None
    base.check(lowbit.matmul(a, b, out=out, accumulate=add), a, b, over, before)
    out.fill_(-7.0)
    assert (whole == -7.0).all()


@pytest.mark.parametrize("pad", [1, 3])
def test_ranges_added_element_by_element(pad):
    m, n, k = 2310, 2401, 9000
    a, b, over = operands("wgrad", m, n, k, 3)
    assert plan(a, b, over, torch.float32).pairs
    whole = torch.full((m, n + pad), 2.0, device="cuda")
    out = whole[:, pad:]
    before = out.double().cpu().numpy()
    base.check(lowbit.matmul(a, b, out=out, accumulate=True), a, b, over, before)
    assert (whole[:, :pad] == 2.0).all()


@pytest.mark.parametrize("floats", [False, True])
@pytest.mark.parametrize("dtype", TWO)
def test_not_a_number_stays_in_its_row(floats, dtype):
    m, n, k = 2500, 2310, 700
    a, b, over = operands("forward", m, n, k, 6, floats)
    assert plan(a, b, over, dtype).pairs
    a.codes[2301, 699] = 0x7F
    nan = torch.isnan(lowbit.matmul(a, b, dtype=dtype))
    assert nan[2301].all() and not nan[:2301].any() and not nan[2302:].any()


def test_same_answer_every_time():
    for way, m, n, k, floats, dtype in (("forward", 2500, 2310, 700, False, torch.bfloat16), ("wgrad", 2310, 2500, 9000, False, torch.float32), ("forward", 2500, 2310, 700, True, torch.bfloat16)):
        a, b, over = operands(way, m, n, k, 2, floats)
        assert plan(a, b, over, dtype).pairs
        first = lowbit.matmul(a, b, over_rows=over, dtype=dtype)
        for _ in range(5):
            assert torch.equal(lowbit.matmul(a, b, over_rows=over, dtype=dtype), first)
