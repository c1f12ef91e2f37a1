"""Products of random sizes, operand kinds, strides and results against 64-bit sums on the GPU; what surrounds a result stays.
Bound: that of the product's other tests."""
import math
import random

import pytest
import torch

from paper_2608_06812_b200 import binding as ozk
from paper_2608_06812_b200 import lowbit

pytestmark = pytest.mark.gpu


def spread(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def matrix(rng, rows, cols, kind, floats):
    ld = -(-cols // 16) * 16 + 16 * rng.randint(0, 2)
    codes = torch.randint(0, 256, (rows, ld), dtype=torch.uint8, device="cuda")   # the padding too
    codes[(codes & 0x7F) == 0x7F] = 0x3A
    if floats:
        shape = {"rows": (rows, -(-cols // 128)), "tiles": (-(-rows // 128), -(-cols // 128))}[kind]
        scales = torch.randn(shape, device="cuda").exp() * 1e-2
    else:
        shape = {"rows": (-(-cols // 512), rows, 4), "cols": (-(-rows // 512), cols, 4), "tiles": (-(-rows // 128), -(-cols // 128))}[kind]
        scales = torch.randint(115, 128, shape, dtype=torch.uint8, device="cuda")
    return lowbit.Fp8Matrix(codes, scales, rows, cols, kind)


@pytest.mark.parametrize("seed", range(8))
def test_products(seed):
    rng, routes = random.Random(seed), set()
    for i in range(100):
        torch.manual_seed(1000 * seed + i)
        m, n = spread(rng, 1, 5000), spread(rng, 1, 5000)
        k = spread(rng, 1, max(2, min(30000, int(4e10 / (m * n)))))
        floats = rng.random() < 0.35
        kind_a, kind_b = ("rows", "tiles") if floats else (rng.choice(["rows", "cols", "tiles"]), rng.choice(["rows", "cols", "tiles"]))
        over = kind_b == "tiles" and not floats and rng.random() < 0.5
        a_over, b_over = kind_a == "cols" or (kind_a == "tiles" and kind_b == "cols"), kind_b == "cols" or over
        a = matrix(rng, *((k, m) if a_over else (m, k)), kind_a, floats)
        b = matrix(rng, *((k, n) if b_over else (n, k)), kind_b, floats)
        dtype = rng.choice([torch.bfloat16, torch.float32])
        add = dtype == torch.float32 and rng.random() < 0.5
        pad = rng.choice([0, 0, 1, 4, 8])
        whole = torch.randn(m + 2, n + 2 * pad + rng.randint(0, 3), device="cuda").mul(k ** 0.5).to(dtype)
        before, at = whole.clone(), (slice(1, 1 + m), slice(pad, pad + n))
        q = ozk.ozk_fp8_gemm_plan(m, n, k, a._operand[a_over], b._operand[b_over], ozk.OZK_BF16 if dtype == torch.bfloat16 else ozk.OZK_F32)
        routes.add((q.pairs, floats))
        lowbit.matmul(a, b, out=whole[at], over_rows=over, accumulate=add)
        A, B = (x.dequantize().double() for x in (a, b))
        A, B = A.T if a_over else A, B.T if b_over else B
        want, size = A @ B.T, A.abs() @ B.abs().T
        if add:
            want, size = want + before[at].double(), size + before[at].double().abs()
        tol = (k / 32 + 33) * 2.0 ** -23 * size
        low, high = want - tol, want + tol
        if dtype == torch.bfloat16:
            low, high = low.bfloat16().double(), high.bfloat16().double()
        got = whole[at].double()
        what = (i, m, n, k, kind_a, kind_b, over, floats, dtype, add, pad, tuple(whole.shape))
        assert ((got >= low) & (got <= high)).all(), what
        whole[at] = before[at]
        assert torch.equal(whole, before), what
    assert len(routes) == 4
    lowbit.check_async()
