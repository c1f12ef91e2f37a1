"""What the norm and the products by expert refuse before anything touches a GPU, and their host-side arithmetic."""
import ctypes
from types import SimpleNamespace

import pytest
import torch

from paper_2608_06812_b200 import binding as ozk
from paper_2608_06812_b200 import build, lowbit

P = 1 << 20   # an address that nothing follows: the checks come first


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def norm_args(**changes):
    a = dict(rows=4, cols=64, x=P, ldx=64, weight=P, root=P, row_codes=P, row_ld=64, row_scales=P, eps=1e-6, x_type=ozk.OZK_BF16, weight_type=ozk.OZK_F32)
    return ozk.ozk_rms_norm_args(**{**a, **changes})


@pytest.mark.parametrize("changes", [dict(rows=-1), dict(cols=-1), dict(ldx=63), dict(x_type=2), dict(weight_type=-1), dict(eps=-1e-6), dict(eps=float("nan")), dict(x=None), dict(x=P + 1), dict(weight=None),
                                     dict(weight=P + 2), dict(root=P + 2), dict(residual=P, ldr=64, ldt=64), dict(residual=P, ldr=63, total=P, ldt=64), dict(residual=P, ldr=64, total=P, ldt=1),
                                     dict(residual=P, ldr=64, total=P, ldt=64, residual_type=3), dict(y=P, ldy=63), dict(y=P, ldy=64), dict(y=P + 1, ldy=64), dict(residual=P, ldr=64, total=P + 64, ldt=64, residual_type=ozk.OZK_BF16, y=P + 64, ldy=64), dict(row_codes=P + 8), dict(row_ld=72), dict(row_ld=48), dict(row_scales=None),
                                     dict(row_codes=None), dict(row_scales=P + 2), dict(root=None, col_codes=P, col_ld=64, col_scales=P), dict(col_codes=P, col_ld=64), dict(col_codes=P, col_ld=65, col_scales=P)])
def test_norm_arguments(changes):
    assert ozk.ozk_rms_norm(norm_args(**changes)) == ozk.OZK_ERR_INVALID_ARG


def test_norm_limits_and_nothing():
    assert ozk.ozk_rms_norm(norm_args(cols=32769, ldx=32769)) == ozk.OZK_ERR_UNSUPPORTED
    assert ozk.ozk_rms_norm(norm_args(rows=2 ** 31)) == ozk.OZK_ERR_UNSUPPORTED
    assert ozk.ozk_rms_norm(norm_args(x_type=ozk.OZK_F32, residual=P, ldr=64, total=P, ldt=64, residual_type=ozk.OZK_BF16)) == ozk.OZK_ERR_UNSUPPORTED
    for empty in (dict(rows=0), dict(cols=0)):
        assert ozk.ozk_rms_norm(norm_args(x=None, weight=None, row_codes=None, row_scales=None, **empty)) == ozk.OZK_OK
    assert ozk.lib().ozk_rms_norm(None, None) == ozk.OZK_ERR_INVALID_ARG and ozk.lib().ozk_rms_norm_backward(None, None) == ozk.OZK_ERR_INVALID_ARG


@pytest.mark.parametrize("changes", [dict(rows=-1), dict(lddy=63), dict(ldt=63), dict(lddx=63), dict(dy_type=2), dict(total_type=2), dict(weight_type=2), dict(dtotal=P, lddt=63), dict(dy=None), dict(total=P + 2), dict(root=None),
                                     dict(weight=P + 1), dict(dx=None), dict(dtotal=P + 2, lddt=64), dict(dweight=P + 2)])
def test_norm_gradient_arguments(changes):
    a = dict(rows=4, cols=64, dy=P, lddy=64, total=P, ldt=64, root=P, weight=P, dx=P, lddx=64, dy_type=ozk.OZK_BF16, total_type=ozk.OZK_F32, weight_type=ozk.OZK_F32)
    assert ozk.ozk_rms_norm_backward(ozk.ozk_rms_norm_backward_args(**{**a, **changes})) == ozk.OZK_ERR_INVALID_ARG


def test_packed_arguments_are_the_structures():
    """The formats that calls are packed with put every field where the structure has it."""
    for form, cls in ((lowbit._NORM_ARGS, ozk.ozk_rms_norm_args), (lowbit._NORM_GRAD_ARGS, ozk.ozk_rms_norm_backward_args)):
        values = list(range(1, len(cls._fields_) + 1))
        there = cls.from_buffer_copy(form.pack(*values))
        assert [getattr(there, name) for name, _ in cls._fields_] == values


def test_segment_blocks():
    """Enough for any division, and no more than one block too many for the worst."""
    assert [ozk.ozk_fp8_segment_blocks(r, e) for r, e in ((0, 5), (1, 5), (5, 5), (128, 1), (129, 1), (1000, 0), (-1, 2), (2, -1))] == [0, 1, 5, 1, 2, 7, 0, 0]
    for rows in (1, 2, 127, 128, 129, 300, 1000):
        for n in (1, 2, 3, 7):
            worst = min(n, rows)
            lone = [1] * (worst - 1) + [rows - worst + 1]
            assert lowbit.segment_blocks(rows, n) == ozk.ozk_fp8_segment_blocks(rows, n) >= sum(-(-c // 128) for c in lone)


OPERAND = dict(codes=P, ld=64, scales=P, scale_kind=ozk.OZK_SCALE_LINES, contract_rows=0)
EXPERTS = dict(codes=P, ld=64, stride=64 * 32, scales=P, contract_rows=0)


def grouped(rows=9, N=32, K=64, experts=3, offsets=P, C=P, c_type=ozk.OZK_F32, ldc=32, clear=0, status=P, x=None, w=None):
    return ozk.ozk_fp8_grouped_gemm(rows, N, K, ozk.ozk_fp8_operand(**{**OPERAND, **(x or {})}), ozk.ozk_fp8_experts(**{**EXPERTS, **(w or {})}), experts, offsets, C, c_type, ldc, clear, status)


def test_grouped_product_arguments():
    for bad in (dict(rows=-1), dict(N=-1), dict(K=-1), dict(experts=-1), dict(c_type=2), dict(ldc=31), dict(clear=2), dict(C=None), dict(C=P + 2), dict(offsets=None), dict(offsets=P + 2), dict(w=dict(contract_rows=2))):
        assert grouped(**bad) == ozk.OZK_ERR_INVALID_ARG, bad
    for bad in (dict(experts=1025), dict(rows=2 ** 31), dict(N=2 ** 31, ldc=2 ** 31), dict(K=2 ** 31)):
        assert grouped(**bad) == ozk.OZK_ERR_UNSUPPORTED, bad
    assert grouped(rows=0, C=None) == ozk.OZK_OK and grouped(N=0, C=None) == ozk.OZK_OK


def test_segment_product_arguments():
    a = ozk.ozk_fp8_operand(**{**OPERAND, "contract_rows": 1})

    def call(experts=3, M=32, N=32, rows=9, offsets=P, C=P, c_type=ozk.OZK_F32, ldc=32, stride=1024, add=0, status=P, left=a, right=a):
        return ozk.ozk_fp8_segment_gemm(experts, M, N, rows, left, right, offsets, C, c_type, ldc, stride, add, status)

    for bad in (dict(experts=-1), dict(M=-1), dict(N=-1), dict(rows=-1), dict(c_type=5), dict(ldc=31), dict(stride=1000), dict(add=2), dict(C=None), dict(C=P + 1), dict(offsets=None), dict(status=None)):
        assert call(**bad) in (ozk.OZK_ERR_INVALID_ARG, ozk.OZK_ERR_WORKSPACE), bad
    for bad in (dict(experts=1025), dict(c_type=ozk.OZK_BF16, add=1), dict(left=ozk.ozk_fp8_operand(**OPERAND)), dict(right=ozk.ozk_fp8_operand(**{**OPERAND, "contract_rows": 1, "scale_kind": ozk.OZK_SCALE_TILES}))):
        assert call(**bad) == ozk.OZK_ERR_UNSUPPORTED, bad
    assert call(left=ozk.ozk_fp8_operand(**{**OPERAND, "contract_rows": 1, "codes": P + 8})) == ozk.OZK_ERR_INVALID_ARG
    assert call(experts=0, C=None) == ozk.OZK_OK and call(M=0, C=None) == ozk.OZK_OK and call(rows=0, add=1) == ozk.OZK_OK


def test_quantiser_arguments():
    q = lambda **k: ozk.ozk_fp8_quantize_segments(*{**dict(rows=4, cols=64, X=P, x_type=ozk.OZK_BF16, ldx=64, offsets=P, segments=2, rc=None, rl=0, rs=None, cc=P, cl=64, cs=P), **k}.values())  # noqa: E731
    for bad in (dict(segments=-1), dict(offsets=None), dict(offsets=P + 1), dict(cc=None), dict(cl=72), dict(cs=None), dict(rc=P, rl=64), dict(rs=P), dict(ldx=63), dict(x_type=2), dict(X=None)):
        assert q(**bad) == ozk.OZK_ERR_INVALID_ARG, bad
    assert q(segments=0, offsets=None) == ozk.OZK_OK
    e = lambda **k: ozk.ozk_fp8_quantize_experts(*{**dict(n=2, rows=4, cols=64, X=P, x_type=ozk.OZK_BF16, ldx=64, xs=256, codes=P, ld=64, step=256, scales=P), **k}.values())  # noqa: E731
    for bad in (dict(n=-1), dict(step=255), dict(step=128), dict(xs=-1), dict(codes=P + 4), dict(scales=None), dict(ld=48), dict(ldx=32)):
        assert e(**bad) == ozk.OZK_ERR_INVALID_ARG, bad
    assert e(n=65536) == ozk.OZK_ERR_UNSUPPORTED and e(n=0, codes=None) == ozk.OZK_OK


def test_layers_check_shapes_first():
    x, w, offsets = torch.zeros(5, 16), torch.zeros(3, 8, 16), torch.zeros(4, dtype=torch.int32)
    for a, b in ((x[0], w), (x, w[0]), (x[:, :15], w)):
        with pytest.raises(ValueError, match="inputs"):
            lowbit.expert_linear(a, b, offsets)
    for bad in (offsets[:3], offsets.long(), offsets.float(), offsets.repeat(2)[::2]):
        with pytest.raises(ValueError, match="offsets"):
            lowbit.expert_linear(x, w, bad)
    with pytest.raises(ValueError, match="w8"):
        lowbit.expert_linear(x, w, offsets, SimpleNamespace(experts=3, rows=8, cols=15))
    with pytest.raises(ValueError, match="residual"):
        lowbit.norm_linear(x, torch.ones(16), torch.zeros(8, 16), torch.zeros(5, 15))
    kept = SimpleNamespace(rows=8, cols=16, kind="cols", scales=torch.zeros(1, dtype=torch.uint8))
    with pytest.raises(ValueError, match="w8"):
        lowbit.norm_linear(x, torch.ones(16), torch.zeros(8, 16), w8=kept)
    for t in (x, w[0]):
        with pytest.raises(ValueError, match="GPU"):
            lowbit.rms_norm(t, torch.ones(16))
    for t in (torch.zeros(3, 8, 16), torch.zeros(3, 8)):
        with pytest.raises(ValueError):
            lowbit.quantize_experts(t)
    with pytest.raises(ValueError, match="GPU"):
        lowbit.Fp8Experts(torch.zeros(1, 2, 16, dtype=torch.uint8), torch.zeros(1, 1, 1, dtype=torch.uint8), 2, 16)
    with pytest.raises(ValueError, match="GPU"):
        lowbit.Fp8Segments(torch.zeros(128, 16, dtype=torch.uint8), torch.zeros(1, 16, 4, dtype=torch.uint8), 2, 16, 1)
