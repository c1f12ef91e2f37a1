"""The norm and its gradients where thread blocks take three rows and more, one after another: rows on their way to shared memory are refilled, and whatever
alternates has come round.  Every layout of a row (one to sixteen warps, one to four groups of 512 columns a warp), type and alignment, against 64 bits on the GPU.

Bounds as in the tests of single rounds: u = 2^-24; 46 u for roots, 48 u for y, and the gradients' own.
"""
import pytest
import torch

from paper_2608_06812_b200 import lowbit

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
TYPES = [(BF16, None), (BF16, BF16), (BF16, F32), (F32, None), (F32, F32)]
# At once on 148 multiprocessors: 3552 rows of one group of 512 columns, 1184 of three and of five, 888 of eight (gradients 444), 444 of sixteen and seventeen, 296 of 32 and 148 of
# more (FP32: from seventeen groups on).
SIZES = [(11000, 500), (11000, 512), (3100, 1100), (4000, 2055), (2800, 4096), (1400, 8192), (1400, 8196), (900, 16384), (460, 20004), (450, 32768)]
ids = lambda t: "_".join("none" if x is None else str(x)[6:] for x in t)  # noqa: E731


def make(rows, cols, dtype, seed, size=1.0, pad=0, offset=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    whole = torch.full((rows, cols + pad + offset), 3.0e4, dtype=dtype, device="cuda")
    part = whole[:, offset:offset + cols]
    part.copy_(torch.randn(rows, cols, generator=g, device="cuda") * torch.randn(rows, 1, generator=g, device="cuda").mul(1.5).exp() * size)
    return part


VALUES = torch.tensor([(f / 8 * 2.0 ** -6) if e == 0 else (1 + f / 8) * 2.0 ** (e - 7) for e in range(16) for f in range(8)], dtype=torch.float64)


def nearest(z):
    """The E4M3 values nearest to |z| <= 448, ties to the even code."""
    v, size = VALUES[:127].cuda(), z.abs()
    up = torch.searchsorted(v, size).clamp_(1, 126)
    low, high = v[up - 1], v[up]
    return torch.where((size - low > high - size) | ((size - low == high - size) & (up % 2 == 0)), high, low) * z.sign()


def exponents(top):
    """The least e >= -127 with top <= 448 2^e; 0 for 0."""
    e = torch.ceil(torch.log2(top / 448.0))
    e = torch.where(torch.exp2(e - 1) * 448.0 >= top, e - 1, e)
    e = torch.where(torch.exp2(e) * 448.0 < top, e + 1, e)
    return torch.where(top > 0, e.clamp(min=-127), 0.0)


def check_form(q, y, kind):
    axis = 1 if kind == "rows" else 0
    e = q.scale_codes().double() - 127
    parts = torch.stack([p.abs().amax(axis) for p in y.split(128, axis)], axis)
    assert ((e >= exponents(parts * (1 - 48 * U))) & (e <= exponents(parts * (1 + 48 * U)))).all(), kind
    z = y * torch.exp2(-e).repeat_interleave(128, axis).narrow(axis, 0, y.shape[axis])
    codes = q.codes[:, :y.shape[1]].long()
    got = VALUES.cuda()[codes & 0x7F] * (1 - 2 * (codes >> 7))
    a, b = (nearest((z * f).clamp(-448.0, 448.0)) for f in (1 - 48 * U, 1 + 48 * U))
    bad = (got < torch.minimum(a, b)) | (got > torch.maximum(a, b))
    assert not bad.any(), (kind, int(bad.sum()), bad.nonzero()[:4])


@pytest.mark.parametrize("types", TYPES, ids=ids)
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("pad,offset", [(0, 0), (4, 4), (1, 0)])
def test_forward(rows, cols, types, pad, offset):
    x = make(rows, cols, types[0], 1, 1.0, pad, offset)
    r = None if types[1] is None else make(rows, cols, types[1], 2, 2.0, pad, offset)
    total = None if r is None else make(rows, cols, types[1], 3, 1.0, pad, offset)
    out = make(rows, cols, types[0], 4, 1.0, pad, offset)
    w = make(1, cols, F32, 5)[0]
    n = lowbit.rms_norm(x, w, r, rows=True, cols=True, y=out, total=total, root=True)
    h = x.double()
    if r is not None:
        h = (x.float() + r.float()).to(r.dtype)
        assert torch.equal(n.total, h)
        h = h.double()
    s = 1.0 / (h.square().mean(1) + 1e-6).sqrt()
    assert ((n.root.double() - s).abs() <= 46 * U * s).all()
    y = h * s[:, None] * w.double()
    half = torch.finfo(types[0]).eps / 2
    assert ((n.y.double() - y).abs() <= y.abs() * (48 * U + half * (1 + 48 * U)) + 1e-38).all()
    check_form(n.rows, y, "rows")
    check_form(n.cols, y, "cols")
    for part in (out, total):   # what lies beside the results stays
        if part is not None:
            part.fill_(3.0e4)
            assert (part._base == 3.0e4).all()


@pytest.mark.parametrize("types", [(BF16, BF16), (BF16, F32), (F32, BF16), (F32, F32)], ids=ids)
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("pad,offset", [(0, 0), (4, 4), (1, 0)])
@pytest.mark.parametrize("add", [False, True])
def test_backward(rows, cols, types, pad, offset, add):
    h, dy = make(rows, cols, types[1], 1, 1.0, pad, offset), make(rows, cols, types[0], 2, 1e-3, pad, offset)
    dh = make(rows, cols, types[1], 3, 1e-3, pad, offset) if add else None
    w = make(1, cols, F32, 5)[0]
    root = (1.0 / (h.double().square().mean(1) + 1e-6).sqrt()).float()
    dx, dw = lowbit.rms_norm_backward(dy, h, root, w, dh)
    s, e = root.double()[:, None], dh.double() if add else torch.zeros((), dtype=torch.float64, device="cuda")
    g, n = dy.double() * w.double(), h.double() * s
    mean, size = (g * n).mean(1, keepdim=True), (g * n).abs().mean(1, keepdim=True)
    want = e + s * (g - n * mean)
    tol = (s * n).abs() * 91 * U * size + 6 * U * (e.abs() + s * (g.abs() + n.abs() * size))
    half = torch.finfo(dx.dtype).eps / 2
    assert ((dx.double() - want).abs() <= tol * (1 + half) + half * want.abs() + 1e-38).all()
    terms = dy.double() * n
    assert ((dw.double() - terms.sum(0)).abs() <= (rows + 42) * U * terms.abs().sum(0) + 1e-38).all()
