"""Quantisation to E4M3 by blocks of 128: codes and scales equal the definition's in 64 bits, bit for bit."""
import numpy as np
import pytest
import torch

from oracle import lowbit as ref
from paper_2608_06812_b200 import lowbit

pytestmark = pytest.mark.gpu


def data(rows, cols, dtype, seed, special=False):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1)) * 3) * np.exp(rng.standard_normal((1, cols)))
    if special and x.size:
        flat = x.reshape(-1)
        at = rng.permutation(x.size)
        for i, v in enumerate((np.nan, np.inf, -np.inf, 0.0, -0.0, 3e38, 1e-38, 1e-44, 448.0, 1.75, np.nextafter(np.float32(1.75), np.float32(2)))):
            flat[at[i % x.size]] = v
        x[rows // 2, :] = 0.0
        x[:, cols // 3] *= 1e-30
    t = torch.from_numpy(x.astype(np.float32)).to(dtype)
    return t, t.double().numpy()


def check(q, exact, kind):
    want, exps = ref.quantize(exact, kind)
    got = q.values8().double().cpu().numpy()
    assert np.array_equal(q.scale_codes().cpu().numpy().astype(np.int64) - 127, exps)
    assert np.array_equal(got, want, equal_nan=True)


SHAPES = [(1, 1), (1, 128), (3, 17), (7, 129), (33, 512), (128, 128), (129, 513), (130, 1040), (257, 255), (5, 2049)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_every_form(rows, cols, dtype):
    x, exact = data(rows, cols, dtype, rows * 1000 + cols, special=rows * cols > 100)
    d = x.cuda()
    r, _ = lowbit.quantize_lines(d)
    check(r, exact, "rows")
    _, c = lowbit.quantize_lines(d, False, True)
    check(c, exact, "cols")
    r2, c2 = lowbit.quantize_lines(d, True, True)
    check(r2, exact, "rows")
    check(c2, exact, "cols")
    check(lowbit.quantize_tiles(d), exact, "tiles")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strided_and_unaligned_input(dtype):
    big, exact = data(70, 700, dtype, 5)
    d = big.cuda()
    for cut in (np.s_[3:69, 1:600], np.s_[::2, 8:520], np.s_[1:, 3:4], np.s_[2:3, 5:]):
        x = d[cut]
        r, c = lowbit.quantize_lines(x, True, True)
        check(r, exact[cut], "rows")
        check(c, exact[cut], "cols")
        check(lowbit.quantize_lines(x)[0], exact[cut], "rows")
        check(lowbit.quantize_tiles(x), exact[cut], "tiles")


def test_nothing_outside_the_matrix_is_written():
    rows, cols, ld = 131, 203, 256
    x, _ = data(rows, cols, torch.bfloat16, 9)
    d = x.cuda()
    for kind in ("rows", "cols", "both", "tiles"):
        q = {}
        for k in ("rows", "cols", "tiles"):
            whole = torch.full((rows + 2, ld), 0xA5, dtype=torch.uint8, device="cuda")
            e = lowbit.Fp8Matrix.empty(rows, cols, k)
            guard = torch.full((e.scales.numel() + 64,), 0xA5, dtype=torch.uint8, device="cuda")
            q[k] = lowbit.Fp8Matrix(whole[1:1 + rows], guard[32:32 + e.scales.numel()].view(e.scales.shape), rows, cols, k), whole, guard
        if kind == "tiles":
            lowbit.quantize_tiles(d, q["tiles"][0])
            used = ("tiles",)
        else:
            lowbit.quantize_lines(d, q["rows"][0] if kind != "cols" else None, q["cols"][0] if kind != "rows" else None)
            used = {"rows": ("rows",), "cols": ("cols",), "both": ("rows", "cols")}[kind]
        for k in used:
            _, whole, guard = q[k]
            w = whole.cpu().numpy()
            assert (w[0] == 0xA5).all() and (w[-1] == 0xA5).all() and (w[:, cols:] == 0xA5).all()
            assert (guard[:32] == 0xA5).all() and (guard[-32:] == 0xA5).all()


def test_unused_scale_bytes_are_one():
    x, _ = data(300, 130, torch.bfloat16, 3)
    r, c = lowbit.quantize_lines(x.cuda(), True, True)
    assert (r.scales[0, :, 2:] == 127).all() and (c.scales[0, :, 3:] == 127).all()
    assert (lowbit.quantize_lines(x.cuda())[0].scales[0, :, 2:] == 127).all()


def test_empty():
    for shape in ((0, 5), (5, 0), (0, 0)):
        r, c = lowbit.quantize_lines(torch.zeros(shape, device="cuda"), True, True)
        assert r.values8().shape == shape and c.values8().shape == shape
        lowbit.quantize_tiles(torch.zeros(shape, device="cuda"))


def test_refusals():
    x = torch.zeros(8, 256, device="cuda")
    for bad in (x.half(), x[0], x.T, x.cpu()):
        with pytest.raises(ValueError):
            lowbit.quantize_lines(bad)
        with pytest.raises(ValueError):
            lowbit.quantize_tiles(bad)
    with pytest.raises(ValueError):
        lowbit.quantize_lines(x, False, False)
    with pytest.raises(ValueError):
        lowbit.quantize_lines(x, lowbit.Fp8Matrix.empty(8, 256, lowbit.COLS))
    with pytest.raises(ValueError):
        lowbit.quantize_tiles(x, lowbit.Fp8Matrix.empty(8, 128, lowbit.TILES))
    codes = torch.zeros(8, 264, dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError):
        lowbit.Fp8Matrix(codes, torch.zeros(1, 8, 4, dtype=torch.uint8, device="cuda"), 8, 256, lowbit.ROWS)
    with pytest.raises(ValueError):
        lowbit.Fp8Matrix(codes[:, :256].contiguous(), torch.zeros(2, 8, 4, dtype=torch.uint8, device="cuda"), 8, 256, lowbit.ROWS)
    with pytest.raises(ValueError):
        lowbit.Fp8Matrix(codes[:, :256].contiguous(), torch.zeros(1, 8, 4, dtype=torch.uint8, device="cuda"), 8, 256, "words")


def test_on_another_stream():
    x, exact = data(513, 640, torch.bfloat16, 21)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        r, c = lowbit.quantize_lines(x.cuda(), True, True)
    s.synchronize()
    check(r, exact, "rows")
    check(c, exact, "cols")
