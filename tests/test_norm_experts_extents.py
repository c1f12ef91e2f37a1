"""How many rows the operators by segments take: row and block indexes are ints.  Refusals come before anything else is looked at, so that a call without
offsets tells them from sizes that are taken (invalid argument)."""
import pytest

from paper_2608_06812_b200 import binding as ozk
from paper_2608_06812_b200 import build

P = 1 << 20   # an address that nothing follows: the checks come first
MOST = 2 ** 31 - 1 - 1024   # rows that are not divided


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def most_rows(experts):
    """The most rows whose blocks of 128 end before 2^31, wherever the segments begin."""
    rows = MOST
    while ozk.ozk_fp8_segment_blocks(rows, experts) * 128 > 2 ** 31 - 1:
        rows -= 1
    return rows


# Blocks begin with each segment: 20 experts of MOST rows may take more than 2^24 of them, the last of which begin beyond 2^31.
@pytest.mark.parametrize("experts", [1, 2, 8, 9, 20, 1024])
def test_blocks_of_segments_stay_within_an_int(experts):
    a = ozk.ozk_fp8_operand(codes=P, ld=16, scales=P, scale_kind=ozk.OZK_SCALE_LINES, contract_rows=1)
    rows = most_rows(experts)
    assert (rows == MOST) == (experts <= 8)
    for r, want in ((rows, ozk.OZK_ERR_INVALID_ARG), (rows + 1, ozk.OZK_ERR_UNSUPPORTED), (MOST + 1, ozk.OZK_ERR_UNSUPPORTED)):
        assert ozk.ozk_fp8_quantize_segments(r, 1, P, ozk.OZK_BF16, 1, None, experts, None, 0, None, P, 16, P) == want
        assert ozk.ozk_fp8_segment_gemm(experts, 1, 1, r, a, a, None, P, ozk.OZK_F32, 1, 1, 0, P) == want


# Rows of nobody are cleared by loops that step over up to 8 rows a multiprocessor: with fewer rows to spare the last step would pass 2^31.
def test_rows_of_grouped_products_leave_room_for_a_step():
    x = ozk.ozk_fp8_operand(codes=P, ld=16, scales=P, scale_kind=ozk.OZK_SCALE_LINES, contract_rows=0)
    w = ozk.ozk_fp8_experts(codes=P, ld=16, stride=16, scales=P, contract_rows=0)
    for rows, want in ((2 ** 31 - 65537, ozk.OZK_ERR_INVALID_ARG), (2 ** 31 - 65536, ozk.OZK_ERR_UNSUPPORTED), (MOST, ozk.OZK_ERR_UNSUPPORTED)):
        for k in (0, 1):
            assert ozk.ozk_fp8_grouped_gemm(rows, 1, k, x, w, 2, None, P, ozk.OZK_BF16, 1, 1, P) == want
