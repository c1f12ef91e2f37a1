"""The 8-bit operators as the first thing that a host thread does with the GPU."""
import threading

import pytest
import torch

from paper_2608_06812_b200 import lowbit
from tests.test_gpu_fp8_gemm import operands

pytestmark = pytest.mark.gpu


def in_a_thread(call):
    """What `call` returns in a new thread, or what it raises there."""
    result = []

    def work():
        try:
            result.append(call())
        except Exception as e:  # noqa: BLE001
            result.append(e)

    t = threading.Thread(target=work)
    t.start()
    t.join()
    if isinstance(result[0], Exception):
        raise result[0]
    return result[0]


@pytest.mark.parametrize("m,n,k", [(3, 300, 512), (2304, 2304, 256)])
def test_product_is_a_threads_first_call(m, n, k):
    a, b, over = operands("forward", m, n, k, 1)
    want = lowbit.matmul(a, b)
    out = torch.zeros_like(want)
    in_a_thread(lambda: lowbit.matmul(a, b, out=out))
    assert torch.equal(out, want)


def test_quantisation_and_adamw_are():
    x = torch.randn(300, 500, device="cuda")
    q, r = lowbit.quantize_tiles(x), lowbit.Fp8Matrix.empty(300, 500, lowbit.TILES)
    in_a_thread(lambda: lowbit.quantize_tiles(x, r))
    assert torch.equal(q.codes[:, :500], r.codes[:, :500]) and torch.equal(q.scales, r.scales)
    p = [torch.ones(1000, device="cuda") for _ in range(2)]
    g = torch.randn(1000, device="cuda")
    tables = [lowbit.AdamWTable.zeros([t], [g]) for t in p]
    tables[0].step(lr=1e-2, step=1)
    torch.cuda.synchronize()
    in_a_thread(lambda: tables[1].step(lr=1e-2, step=1))
    assert torch.equal(p[0], p[1])
