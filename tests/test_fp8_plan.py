"""Which kernel a product takes and what memory it needs, for 148 multiprocessors: decided on the host."""
import pytest

from paper_2608_06812_b200 import binding as ozk
from paper_2608_06812_b200 import build

P = 1 << 20   # an aligned address that is never followed
BF16, F32 = ozk.OZK_BF16, ozk.OZK_F32


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def plan(m, n, k, c_type=BF16, floats=False, a_over=0, b_over=0, sms=148):
    up = lambda x: -(-x // 16) * 16  # noqa: E731
    a = ozk.ozk_fp8_operand(P, up(m if a_over else k), P, 2 if floats else 0, a_over)
    b = ozk.ozk_fp8_operand(P, up(n if b_over else k), P, 3 if floats else 0 if b_over else 1, b_over)
    return ozk.ozk_fp8_gemm_plan(m, n, k, a, b, c_type, sms)


def test_few_rows_take_clusters_and_need_no_memory():
    for m, n, k, tile, splits in ((1, 4096, 4096, 16, 8), (17, 512, 384, 32, 1), (64, 16384, 4096, 64, 2), (128, 128, 128, 128, 1)):
        q = plan(m, n, k)
        assert (q.pairs, q.tile_rows, q.tile_cols, q.splits, q.scratch_bytes) == (0, tile, 128, splits, 0)
        assert q.tiles == -(-n // 128)


def test_many_tiles_take_pairs_with_whole_sums():
    for m, n, k in ((8192, 8192, 8192), (2304, 2304, 700), (384, 8192, 4096)):
        q = plan(m, n, k)
        assert (q.pairs, q.tile_rows, q.tile_cols, q.splits, q.scratch_bytes) == (1, 256, 256, 1, 0)
        assert q.tiles == -(-m // 256) * -(-n // 256)


def test_split_sums_pass_through_memory():
    for args, splits in ((dict(m=512, n=2048, k=8192, floats=True), 4), (dict(m=1024, n=1024, k=16384, floats=True), 4), (dict(m=256, n=256, k=40000, c_type=F32), 39),
                         (dict(m=300, n=301, k=40000, c_type=F32, a_over=1, b_over=1), 18)):
        q = plan(**args)
        assert (q.pairs, q.splits) == (1, splits)
        assert q.scratch_bytes == splits * args["m"] * -(-args["n"] // 4) * 4 * 4
        assert q.scratch_bytes <= ozk.ozk_fp8_gemm_workspace_bytes() - 1024


def test_empty_products_and_refusals():
    for shape in ((0, 5, 5), (5, 0, 5), (5, 5, 0)):
        q = plan(*shape)
        assert (q.pairs, q.tiles, q.splits, q.scratch_bytes) == (0, 0, 0, 0)
    for bad in (dict(m=-1, n=1, k=1), dict(m=1, n=1, k=1, c_type=5), dict(m=1, n=1, k=1, sms=-1), dict(m=1 << 31, n=1, k=1), dict(m=1, n=1, k=1, floats=True, b_over=1)):
        with pytest.raises(ozk.OzkError):
            plan(**bad)


def test_scratch_refusals():
    a, b = ozk.ozk_fp8_operand(P, 128, P, 0, 0), ozk.ozk_fp8_operand(P, 128, P, 0, 0)
    call = lambda c=P, status=P, scratch=None, acc=0, ldc=8: ozk.ozk_fp8_gemm_scratch(8, 8, 128, a, b, c, BF16, ldc, acc, status, scratch)  # noqa: E731
    assert call(status=None) == ozk.OZK_ERR_WORKSPACE
    assert call(status=P + 128) == call(scratch=P + 16) == call(c=None) == call(c=P + 1) == call(ldc=7) == call(acc=2) == ozk.OZK_ERR_INVALID_ARG
    assert call(acc=1) == ozk.OZK_ERR_UNSUPPORTED
