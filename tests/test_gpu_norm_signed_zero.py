"""The norm's codes are those that quantize_lines writes for its answer, byte for byte: a negative zero keeps its sign beside a NaN or an infinity too."""
import pytest
import torch

from paper_2608_06812_b200 import lowbit

pytestmark = pytest.mark.gpu


def stream(rows, cols, dtype, shift):
    """Many zeros of both signs, a NaN and an infinity in rows and columns of their own; rows at odd places with `shift`."""
    g = torch.Generator().manual_seed(rows + cols)
    x = torch.randn(rows, cols, generator=g)
    x = torch.where(torch.rand(rows, cols, generator=g) < 0.3, torch.where(torch.rand(rows, cols, generator=g) < 0.5, 0.0, -0.0), x)
    x[rows // 2, cols // 3] = float("nan")
    x[rows // 4, cols - 1] = float("inf")
    whole = torch.zeros(rows, cols + shift, dtype=dtype, device="cuda")
    whole[:, shift:] = x.to(dtype)
    return whole[:, shift:]


@pytest.mark.parametrize("rows,cols", [(9, 1024), (130, 1024), (260, 700), (5, 515)])
@pytest.mark.parametrize("shift", [0, 1, 4])
def test_codes_are_the_quantisers(rows, cols, shift):
    x = stream(rows, cols, torch.float32, shift)
    w = torch.linspace(-2.0, 2.0, cols, device="cuda")
    n = lowbit.rms_norm(x, w, rows=True, cols=True, y=True)
    by_rows, by_cols = lowbit.quantize_lines(n.y, True, True)
    for got, want in ((n.rows, by_rows), (n.cols, by_cols)):
        assert torch.equal(got.codes[:, :cols] & 0x7F, want.codes[:, :cols] & 0x7F) and torch.equal(got.scales, want.scales)
        number = (want.codes[:, :cols] & 0x7F) != 0x7F   # the sign of a NaN means nothing
        assert torch.equal(got.codes[:, :cols][number], want.codes[:, :cols][number])


@pytest.mark.parametrize("residual", [None, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(9, 1024), (130, 1024), (260, 700), (5, 515)])
@pytest.mark.parametrize("shift", [0, 1, 4])
def test_zeros_of_bfloat16_keep_their_sign(rows, cols, shift, residual):
    x = stream(rows, cols, torch.bfloat16, shift)
    r = None if residual is None else x.to(residual)   # x + x: zeros, NaN and infinities where x has them
    w = torch.linspace(-2.0, 2.0, cols, device="cuda")
    n = lowbit.rms_norm(x, w, r, rows=True, cols=True, y=True)
    row_ok = torch.isfinite(x.float()).all(1)          # a root of zero or NaN makes other zeros or none
    zero = (x == 0) & row_ok[:, None]
    want = torch.where(torch.signbit(n.y), 0x80, 0x00).to(torch.uint8)
    assert zero.any() and torch.equal(torch.signbit(n.y)[zero], (torch.signbit(x.float()) ^ torch.signbit(w))[zero])
    for q in (n.rows, n.cols):
        assert torch.equal(q.codes[:, :cols][zero], want[zero])
