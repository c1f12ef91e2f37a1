"""Codes of negative zeros beside what is not finite: the sign stays, and all forms write the same bytes."""
import numpy as np
import pytest
import torch

from paper_2608_06812_b200 import lowbit

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantised(dtype):
    g = torch.Generator().manual_seed(0)
    x = torch.randn(300, 700, generator=g)
    x[torch.rand(300, 700, generator=g) < 0.2] = -0.0
    x[torch.rand(300, 700, generator=g) < 0.1] = 0.0
    x[torch.rand(300, 700, generator=g) < 0.01] = float("nan")
    x[torch.rand(300, 700, generator=g) < 0.01] = float("-inf")
    d = x.to(dtype).cuda()
    both = lowbit.quantize_lines(d, True, True)
    forms = [lowbit.quantize_lines(d)[0], lowbit.quantize_lines(d, False, True)[1], *both, lowbit.quantize_tiles(d)]
    zero, sign, nan = (x == 0).numpy(), np.signbit(x.numpy()), ~np.isfinite(x.numpy())
    for q in forms:
        codes = q.codes.cpu().numpy()[:, :700]
        assert (codes[zero] == np.where(sign[zero], 0x80, 0)).all()
        assert ((codes[nan] & 0x7F) == 0x7F).all()
    same = lambda a, b: torch.equal(a.codes[:, :700], b.codes[:, :700])  # noqa: E731
    assert same(forms[0], both[0]) and same(forms[1], both[1])


def test_first_moments():
    p, g = torch.ones(128, device="cuda"), torch.full((128,), -0.0, device="cuda")
    g[5], g[6] = float("nan"), 1.0
    t = lowbit.AdamWTable.zeros([p], [g])
    t.tensors["m"][0].fill_(0x80)
    t.step(lr=1e-3, step=1)
    m = t.tensors["m"][0].cpu().numpy()
    assert (m[5] & 0x7F) == 0x7F and 0 < m[6] < 0x7F and (np.delete(m, [5, 6]) == 0x80).all()
