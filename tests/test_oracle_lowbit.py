"""Pins of the oracle of the 8-bit operators, and refusals of their entry points that need no GPU."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import lowbit as ref
from paper_2608_06812_b200 import binding as ozk
from paper_2608_06812_b200 import build


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def test_e4m3_values_are_those_of_torch():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.decode(codes), want, equal_nan=True)


def test_nearest_agrees_with_torch_on_every_half_step():
    grid = ref.E4M3[:127]
    x = np.concatenate([grid, (grid[1:] + grid[:-1]) / 2, np.nextafter(np.float32((grid[1:] + grid[:-1]) / 2), np.float32(1e9)).astype(np.float64)])
    x = np.concatenate([x, -x])
    want = torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.nearest(x), want)
    assert np.isnan(ref.nearest(np.array([np.inf, -np.inf, np.nan]))).all()


def test_scale_exponent_is_the_least_that_fits():
    rng = np.random.default_rng(0)
    for amax in np.concatenate([2.0 ** rng.uniform(-118, 119, 300), [448.0, 448.0 * 2.0 ** -20, 449.0, np.nextafter(448.0, 449.0), 1.75 * 2.0 ** 100]]):
        e = ref.scale_exponent(np.array([0.0, -amax, np.nan, np.inf]))
        assert 448.0 * 2.0 ** e >= amax > 448.0 * 2.0 ** (e - 1)
    assert ref.scale_exponent(np.zeros(3)) == 0
    assert ref.scale_exponent(np.array([1e-45])) == -127


def test_stochastic_roots_are_unbiased_and_never_zero():
    y = np.full(128, 5.3)
    bits = np.arange(65536)[::512]
    w = ref.root_values(y * 2.0 ** -3, np.array([-3]), bits)
    assert set(w) == {5.0, 5.5} and abs(w.mean() - 5.3) < 0.01
    assert (ref.root_values(np.full(128, 1e-9), np.array([0])) == 2.0 ** -9).all()


def test_line_scale_bytes():
    assert ozk.ozk_fp8_line_scale_bytes(10, 512) == 40
    assert ozk.ozk_fp8_line_scale_bytes(10, 513) == 80
    assert ozk.ozk_fp8_line_scale_bytes(10, 0) == 0
    assert ozk.ozk_fp8_line_scale_bytes(-1, 5) == 0


P = 1 << 20   # an aligned address that is never followed: every call below is refused before it is used


def lines(rows=4, cols=64, X=P, kind=ozk.OZK_BF16, ldx=64, q=P, ld=64, s=P, qc=None, ldc=0, sc=None):
    return ozk.ozk_fp8_quantize_lines(rows, cols, X, kind, ldx, q, ld, s, qc, ldc, sc)


@pytest.mark.parametrize("change", [dict(rows=-1), dict(ldx=63), dict(kind=2), dict(X=None), dict(X=P + 1), dict(q=P + 8), dict(ld=60), dict(ld=48), dict(s=P + 1),
                                    dict(s=None), dict(q=None, s=None), dict(q=None), dict(qc=P, ldc=72, sc=P), dict(qc=P, ldc=64)])
def test_quantize_refusals(change):
    assert lines(**change) == ozk.OZK_ERR_INVALID_ARG


def test_quantize_limits_and_empty():
    assert lines(rows=1 << 31) == ozk.OZK_ERR_UNSUPPORTED
    assert lines(rows=0) == ozk.OZK_OK and lines(cols=0) == ozk.OZK_OK
    tiles = lambda **k: ozk.ozk_fp8_quantize_tiles(*{**dict(rows=4, cols=64, X=P, kind=0, ldx=64, q=P, ld=64, s=P), **k}.values())  # noqa: E731
    assert tiles(rows=0) == ozk.OZK_OK
    assert tiles(q=P + 1) == tiles(ld=65) == tiles(s=None) == tiles(X=P + 2) == ozk.OZK_ERR_INVALID_ARG


def operand(codes=P, ld=128, scales=P, kind=0, over=0):
    return ozk.ozk_fp8_operand(codes, ld, scales, kind, over)


def gemm(M=8, N=8, K=128, A=None, B=None, C=P, ctype=1, ldc=8, acc=0, ws=P, wsb=1 << 30):
    return ozk.ozk_fp8_gemm(M, N, K, A or operand(), B or operand(), C, ctype, ldc, acc, ws, wsb)


@pytest.mark.parametrize("change", [dict(M=-1), dict(N=-1), dict(K=-1), dict(ldc=7), dict(C=None), dict(C=P + 1), dict(ctype=2), dict(acc=2), dict(ws=P + 128),
                                    dict(A=operand(codes=P + 8)), dict(A=operand(ld=120)), dict(A=operand(ld=112)), dict(B=operand(scales=None)), dict(B=operand(kind=4)),
                                    dict(B=operand(over=2)), dict(A=operand(scales=P + 2)), dict(B=operand(codes=None))])
def test_gemm_refusals(change):
    assert gemm(**change) == ozk.OZK_ERR_INVALID_ARG


@pytest.mark.parametrize("change", [dict(acc=1), dict(M=1 << 31, ldc=8), dict(A=operand(kind=2)), dict(B=operand(kind=3)), dict(A=operand(kind=2), B=operand(kind=2)),
                                    dict(A=operand(kind=2, over=1), B=operand(kind=3)), dict(A=operand(kind=3), B=operand(kind=3))])
def test_gemm_unsupported(change):
    assert gemm(**change) == ozk.OZK_ERR_UNSUPPORTED


def test_gemm_workspace():
    need = ozk.ozk_fp8_gemm_workspace_bytes()
    assert gemm(wsb=need - 1) == ozk.OZK_ERR_WORKSPACE
    ozk.ozk_set_workspace(None, 0)
    assert gemm(ws=None) == ozk.OZK_ERR_WORKSPACE
    assert ozk.ozk_get_workspace_status(None) == ozk.OZK_ERR_WORKSPACE
    assert gemm(M=0) == ozk.OZK_OK and gemm(N=0) == ozk.OZK_OK


def adamw(count=1, n=10, param=P, grad=P, m=P, v=P, ms=P, vs=P, copy=None, **options):
    o = dict(param_type=0, grad_type=1, state_bits=8, stochastic=0, seed=0, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, step=1, grad_scale=None, skip=None)
    o.update(options)
    table = (ozk.ozk_adamw_tensor * 1)(ozk.ozk_adamw_tensor(param, grad, m, v, ms, vs, copy, n))
    return ozk.ozk_adamw_step(ctypes.byref(table), count, ozk.ozk_adamw_options(*o.values()))


@pytest.mark.parametrize("change", [dict(count=-1), dict(n=-1), dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(ms=None), dict(vs=None),
                                    dict(param=P + 2), dict(grad=P + 1), dict(state_bits=16), dict(stochastic=2), dict(step=0), dict(param_type=2), dict(grad_type=-1),
                                    dict(beta1=1.0), dict(beta2=-0.1), dict(eps=float("nan")), dict(lr=-1.0), dict(weight_decay=float("nan")), dict(grad_scale=P + 1), dict(skip=P + 2),
                                    dict(param_type=1, copy=P), dict(copy=P + 1), dict(state_bits=32, m=P + 1)])
def test_adamw_refusals(change):
    assert adamw(**change) == ozk.OZK_ERR_INVALID_ARG


def test_adamw_limits():
    assert adamw(n=1 << 50) == ozk.OZK_ERR_UNSUPPORTED
