"""Blocks that hold a NaN or an infinity, in every layout of the norm: the others' codes and scales are the formula's.

Rows with a NaN answer NaN, rows with an infinity zeros (and NaN for itself); weights that are not finite leave the rest of each row as it is, so that blocks by rows
and by columns have finite entries of full size beside what is not.  One column's largest entry lies above the largest BF16 number.  Bounds as in the tests of finite numbers.
"""
import numpy as np
import pytest
import torch

from paper_2608_06812_b200 import lowbit
from tests.test_gpu_norm import BF16, F32, TYPES, U, check_form, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("types", TYPES, ids=lambda t: "_".join("none" if x is None else str(x)[6:] for x in t))
@pytest.mark.parametrize("rows,cols", [(9, 1024), (130, 1024), (260, 700), (131, 1030), (8, 4096), (6, 8196), (6, 16384), (6, 20004)])
@pytest.mark.parametrize("pad,offset", [(0, 0), (4, 4), (1, 0), (2, 1)])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_what_is_not_finite_leaves_the_rest(rows, cols, types, pad, offset, eps):
    x = make(rows, cols, types[0], rows + cols, pad=pad, offset=offset)
    r = None if types[1] is None else make(rows, cols, types[1], rows + cols + 1, 2.0, pad, offset)
    large = cols // 2 + 3   # a column with one entry, in the row of ones
    for t in (x,) if r is None else (x, r):
        t[:, large] = 0.0
        t[1] = 1.0 if r is None else 0.5
        t[0] = -0.0
    x[2, 5], x[3, cols - 1], x[rows - 1, cols // 3], x[rows - 2, 600] = float("nan"), float("inf"), float("-inf"), float("nan")
    w = make(1, cols, F32, 3)[0]
    w[large], w[7], w[cols - 2], w[130] = 3.4e38, float("nan"), float("inf"), float("-inf")
    n = lowbit.rms_norm(x, w, r, eps=eps, rows=True, cols=True, root=True)
    h = (x if r is None else (x.float() + r.float()).to(r.dtype)).double().cpu().numpy()
    with np.errstate(all="ignore"):
        s = 1.0 / np.sqrt((h * h).mean(1) + float(np.float32(eps)))
        y = h * s[:, None] * w.double().cpu().numpy()
    y[~np.isfinite(y)] = np.nan   # codes of infinities are NaN
    root = n.root.double().cpu().numpy()
    finite = np.isfinite(s)
    assert np.array_equal(np.isnan(root), np.isnan(s)) and np.array_equal(np.isinf(root), np.isinf(s)) and (np.abs(root[finite] - s[finite]) <= 46 * U * s[finite]).all()
    assert abs(y[1, large]) > 3.39e38
    check_form(n.rows, y, "rows")
    check_form(n.cols, y, "cols")


@pytest.mark.parametrize("rows,cols", [(130, 1024), (140, 700), (5, 515)])
@pytest.mark.parametrize("shift", [0, 1])
def test_rows_of_bfloat16_of_any_bits(rows, cols, shift):
    """Most rows hold a NaN or an infinity; the finite ones are as large as the type goes, or as small."""
    g = torch.Generator().manual_seed(rows)
    bits = torch.randint(-2 ** 15, 2 ** 15, (rows, cols + shift), generator=g, dtype=torch.int16)
    bits[::3] &= 0x3FFF - 2 ** 15            # no infinities, below two: squares within FP32, many below it
    x = bits.view(BF16).cuda()[:, shift:]
    w = make(1, cols, BF16, 3)[0]
    n = lowbit.rms_norm(x, w, rows=True, cols=True, root=True)
    h = x.double().cpu().numpy()
    with np.errstate(all="ignore"):
        y = h * n.root.double().cpu().numpy()[:, None] * w.double().cpu().numpy()   # the roots are held to the formula elsewhere
    y[~np.isfinite(y)] = np.nan
    assert np.isfinite(y).all(1).any() and not np.isfinite(y).all()
    check_form(n.rows, y, "rows")
    check_form(n.cols, y, "cols")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cols", [300, 4096, 20004])
def test_sums_of_squares_at_the_end_of_float32(dtype, cols):
    """Beyond it they count as infinite, whatever their mean; up to half of it the answer is the formula's."""
    most = float(np.finfo(np.float32).max)
    below, above = 2.0 ** np.floor(np.log2((most / 2 / cols) ** 0.5)), 2.0 ** np.ceil(np.log2((most * 2 / cols) ** 0.5))
    x = torch.tensor([below, above], device="cuda").to(dtype)[:, None].repeat(1, cols)
    n = lowbit.rms_norm(x, torch.ones(cols, device="cuda"), rows=True, cols=True, y=True, root=True)
    assert (n.root[0] * below - 1).abs() <= 46 * U and (n.y[0] == 1).all() and (n.rows.dequantize()[0] == 1).all()
    assert n.root[1] == 0 and (n.y[1] == 0).all() and (n.rows.dequantize()[1] == 0).all() and (n.cols.dequantize() == torch.tensor([[1.0], [0.0]], device="cuda")).all()
