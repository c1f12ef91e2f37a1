"""Refusals of `lowbit` that come before anything touches a GPU."""
from types import SimpleNamespace

import pytest

from paper_2608_06812_b200 import lowbit


def matrix(rows, cols, kind):
    return SimpleNamespace(rows=rows, cols=cols, kind=kind, index=0)


def test_a_matrix_by_rows_is_not_summed_over_its_rows():
    """The switch would be ignored: with a square b the result is a b^T where a b was asked for."""
    with pytest.raises(ValueError, match="by rows"):
        lowbit.matmul(matrix(4, 8, "rows"), matrix(8, 8, "rows"), over_rows=True)
