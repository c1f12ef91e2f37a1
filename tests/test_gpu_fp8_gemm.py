"""The block-scaled product against 64-bit sums of the same scaled values.

Bound of an FP32 sum on the tensor cores, from their accumulation: each instruction adds 32 products, cut off (not
rounded) at the last place of the largest term, to a running sum that is cut off once: at most (K / 32 + 33) units of
2^-23 of S = sum_k |a b|.  Sums over ranges and tiles are joined by FP32 additions, 2^-24 S each and fewer.  A BF16
result lies between the roundings of the two ends of that interval.
"""
import numpy as np
import pytest
import torch

from oracle import lowbit as ref
from paper_2608_06812_b200 import binding as ozk
from paper_2608_06812_b200 import lowbit

pytestmark = pytest.mark.gpu


def values(m):
    """The scaled values of an Fp8Matrix in 64 bits, by the oracle."""
    codes = ref.decode(m.codes.cpu().numpy()[:, :m.cols])
    s = m.scale_codes().cpu().numpy()
    s = s.astype(np.float64) if s.dtype == np.float32 else 2.0 ** (s.astype(np.float64) - 127.0)
    return codes * ref.spread(s, codes.shape, m.kind)


def random_matrix(rows, cols, kind, seed, floats=False):
    """Random codes (no NaN), scales over 12 binades."""
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 256, (rows, -(-max(cols, 1) // 16) * 16), generator=g, dtype=torch.uint8)
    codes[(codes & 0x7F) == 0x7F] = 0x3A
    e = lowbit.Fp8Matrix.empty(rows, cols, kind)
    if floats:
        shape = {"rows": (rows, -(-cols // 128)), "tiles": (-(-rows // 128), -(-cols // 128))}[kind]
        scales = torch.randn(shape, generator=g).exp().mul(1e-2)
    else:
        scales = torch.randint(115, 128, tuple(e.scales.shape), generator=g, dtype=torch.uint8)
    return lowbit.Fp8Matrix(codes.cuda(), scales.cuda(), rows, cols, kind)


def operands(way, m, n, k, seed, floats=False):
    if way == "forward":
        return random_matrix(m, k, "rows", seed, floats), random_matrix(n, k, "tiles", seed + 1, floats), False
    if way == "dgrad":
        return random_matrix(m, k, "rows", seed), random_matrix(k, n, "tiles", seed + 1), True
    if way == "wgrad":
        return random_matrix(k, m, "cols", seed), random_matrix(k, n, "cols", seed + 1), False
    if way == "lines":          # both operands by rows
        return random_matrix(m, k, "rows", seed), random_matrix(n, k, "rows", seed + 1), False
    if way == "mixed":          # tiles on the left, summed over its rows; lines on the right
        return random_matrix(k, m, "tiles", seed), random_matrix(k, n, "cols", seed + 1), False
    raise AssertionError(way)


def check(c, a, b, over_rows, before=None):
    A, B = values(a), values(b)
    A = A.T if a.kind == "cols" or (a.kind == "tiles" and b.kind == "cols") else A
    B = B.T if b.kind == "cols" or (b.kind == "tiles" and over_rows) else B
    want, size = A @ B.T, np.abs(A) @ np.abs(B).T
    if before is not None:
        want, size = want + before, size + np.abs(before)
    K = A.shape[1]
    tol = (K / 32 + 33) * 2.0 ** -23 * size
    low, high = want - tol, want + tol
    if c.dtype == torch.bfloat16:
        low, high = (torch.from_numpy(x).bfloat16().double().numpy() for x in (low, high))
    got = c.double().cpu().numpy()
    assert got.shape == want.shape
    bad = ~((got >= low) & (got <= high))
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4], np.abs(got - want).max())


# on both sides of every choice between the kernels, tile widths and splits of K
SIZES = [(1, 1, 1), (1, 16, 128), (1, 257, 300), (2, 130, 1024), (16, 64, 640), (17, 512, 384), (33, 200, 129), (64, 384, 2048), (61, 1000, 777), (100, 300, 520),
         (128, 128, 128), (129, 128, 640), (200, 264, 1000), (256, 256, 512), (257, 255, 1100), (300, 520, 2050), (700, 17, 260), (513, 1025, 96)]


@pytest.mark.parametrize("way", ["forward", "dgrad", "wgrad", "lines", "mixed"])
@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_product(way, m, n, k, dtype):
    a, b, over = operands(way, m, n, k, m + n + k)
    check(lowbit.matmul(a, b, over_rows=over, dtype=dtype), a, b, over)
    lowbit.check_async()


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_float_scales(m, n, k, dtype):
    a, b, _ = operands("forward", m, n, k, 7 * m + n + k, floats=True)
    check(lowbit.matmul(a, b, dtype=dtype), a, b, False)
    lowbit.check_async()


@pytest.mark.parametrize("way", ["forward", "dgrad", "wgrad"])
@pytest.mark.parametrize("m,n,k", [(1, 100, 300), (64, 256, 256), (130, 260, 520), (512, 512, 4096), (300, 300, 20000)])
def test_accumulate(way, m, n, k):
    a, b, over = operands(way, m, n, k, m + n + k)
    c = torch.randn(m, n, generator=torch.Generator().manual_seed(1)).mul(float(k) ** 0.5).cuda()
    before = c.double().cpu().numpy()
    got = lowbit.matmul(a, b, out=c, over_rows=over, accumulate=True)
    assert got.data_ptr() == c.data_ptr()
    check(c, a, b, over, before)
    lowbit.check_async()


@pytest.mark.parametrize("m,n,k", [(40, 100, 12000), (130, 700, 3000), (512, 512, 8192), (260, 256, 1024), (1, 4096, 4096), (5, 8192, 512), (1024, 1024, 16384), (4096, 300, 256), (130, 4100, 8190), (2048, 2048, 9000)])
@pytest.mark.parametrize("way", ["forward", "dgrad", "wgrad"])
def test_larger(way, m, n, k):
    a, b, over = operands(way, m, n, k, 3)
    check(lowbit.matmul(a, b, over_rows=over, dtype=torch.float32), a, b, over)
    if way == "forward":
        a, b, _ = operands(way, m, n, k, 4, floats=True)
        check(lowbit.matmul(a, b), a, b, False)
    lowbit.check_async()


def test_long_sums_in_32_bits_keep_their_precision():
    """Over 16384 and more, ranges of 8192 joined in FP32: under 2e-6 of the result's norm (measured 1.2e-6 without ranges at 16384, growing)."""
    a, b, _ = operands("wgrad", 256, 256, 40000, 11)
    c = lowbit.matmul(a, b, dtype=torch.float32).double().cpu().numpy()
    want = values(a).T @ values(b)
    assert np.linalg.norm(c - want) < 2e-6 * np.linalg.norm(want)


@pytest.mark.parametrize("dtype,pad", [(torch.bfloat16, 1), (torch.bfloat16, 3), (torch.float32, 1), (torch.float32, 4), (torch.bfloat16, 8)])
def test_strided_output_leaves_its_surroundings(dtype, pad):
    for m, n, k in ((37, 200, 256), (300, 333, 512), (1, 50, 2000)):
        a, b, over = operands("forward", m, n, k, 5)
        whole = torch.full((m + 2, n + 2 * pad), -7.0, dtype=dtype, device="cuda")
        out = whole[1:1 + m, pad:pad + n]
        check(lowbit.matmul(a, b, out=out), a, b, over)
        out.fill_(-7.0)
        assert (whole == -7.0).all()


def test_not_a_number_stays_in_its_row():
    for m, n, k in ((5, 300, 512), (300, 300, 512)):
        for floats in (False, True):
            a, b, over = operands("forward", m, n, k, 6, floats)
            a.codes[2, 100] = 0x7F
            c = lowbit.matmul(a, b, dtype=torch.float32)
            nan = torch.isnan(c)
            assert nan[2].all() and not nan[:2].any() and not nan[3:].any()


def test_rows_of_zeros_and_extreme_scales():
    m, n, k = 40, 300, 384
    a, b, over = operands("forward", m, n, k, 8)
    a.codes[3] = 0
    a.codes[4] = 0x80
    a.scales[:, 5] = 0          # 2^-127
    a.scales[:, 6] = 200        # 2^73
    c = lowbit.matmul(a, b, dtype=torch.float32)
    assert (c[3] == 0).all() and (c[4] == 0).all()
    want = values(a) @ values(b).T
    got = c.double().cpu().numpy()
    assert np.allclose(got[6], want[6], rtol=1e-4, atol=1e-5 * np.abs(want[6]).max())
    assert np.abs(got[5]).max() < 1e-30


def test_empty():
    for m, n, k in ((0, 5, 5), (5, 0, 5), (5, 7, 0), (300, 300, 0)):
        a, b, over = operands("forward", m, n, k, 1)
        c = lowbit.matmul(a, b, dtype=torch.float32)
        assert c.shape == (m, n) and (c == 0).all()
    a, b, over = operands("forward", 5, 7, 0, 1)
    c = torch.ones(5, 7, device="cuda")
    lowbit.matmul(a, b, out=c, accumulate=True)
    assert (c == 1).all()


def test_same_answer_every_time():
    for way, m, n, k in (("forward", 7, 4096, 4096), ("wgrad", 300, 300, 20000), ("forward", 512, 512, 8192)):
        a, b, over = operands(way, m, n, k, 2)
        first = lowbit.matmul(a, b, over_rows=over, dtype=torch.float32)
        for _ in range(5):
            assert torch.equal(lowbit.matmul(a, b, over_rows=over, dtype=torch.float32), first)


def test_two_streams_at_once():
    jobs = [operands("forward", 64, 2048, 4096, 1), operands("wgrad", 512, 512, 8000, 2)]
    want = [lowbit.matmul(a, b, over_rows=o, dtype=torch.float32) for a, b, o in jobs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, (a, b, o) in enumerate(jobs):
            with torch.cuda.stream(streams[i]):
                got[i].append(lowbit.matmul(a, b, over_rows=o, dtype=torch.float32))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(c, want[i]) for c in got[i])


def test_in_a_graph():
    jobs = [(*operands("forward", 3, 1000, 2048, 1), torch.empty(3, 1000, device="cuda")), (*operands("wgrad", 300, 260, 9000, 2), torch.empty(300, 260, device="cuda"))]
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for a, b, o, c in jobs:
            lowbit.matmul(a, b, out=c, over_rows=o)
    s.synchronize()
    want = [c.clone() for *_, c in jobs]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        for a, b, o, c in jobs:
            lowbit.matmul(a, b, out=c, over_rows=o)
    for *_, c in jobs:
        c.zero_()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(w, c) for w, (*_, c) in zip(want, jobs))


def test_registered_workspace_serves_too():
    ws = torch.zeros(ozk.ozk_fp8_gemm_workspace_bytes(), dtype=torch.uint8, device="cuda")
    ozk.check(ozk.ozk_set_workspace(ws.data_ptr(), ws.numel()), "ozk_set_workspace")
    a, b, over = operands("forward", 20, 300, 700, 9)
    c = torch.empty(20, 300, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    ozk.check(ozk.ozk_fp8_gemm(20, 300, 700, a._operand[0], b._operand[0], c.data_ptr(), ozk.OZK_F32, 300, stream=s), "ozk_fp8_gemm")
    ozk.check(ozk.ozk_get_async_status(s), "status")
    check(c, a, b, over)
    ozk.ozk_set_workspace(None, 0)
    from tests import gpu_util
    gpu_util._ws["buf"] = None


def test_refusals():
    a, b, _ = operands("forward", 4, 32, 256, 1)
    for call in (lambda: lowbit.matmul(a, random_matrix(32, 255, "tiles", 1)), lambda: lowbit.matmul(a, b, dtype=torch.float16), lambda: lowbit.matmul(a, b, accumulate=True),
                 lambda: lowbit.matmul(a, b, out=torch.empty(32, 4, device="cuda")), lambda: lowbit.matmul(a, b, out=torch.empty(32, 4, device="cuda").T),
                 lambda: lowbit.matmul(a, b, out=torch.empty(4, 32)), lambda: lowbit.matmul(a, b, out=torch.empty(4, 32, device="cuda", dtype=torch.float64))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ozk.OzkError):
        lowbit.matmul(a, b, out=torch.zeros(4, 32, device="cuda", dtype=torch.bfloat16), accumulate=True)
    with pytest.raises(ozk.OzkError):
        lowbit.matmul(random_matrix(4, 256, "rows", 1, floats=True), b)
