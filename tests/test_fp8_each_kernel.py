"""Each kernel of the 8-bit floating-point linear in both 16-bit types, with and without ReLU, and the norm at row counts and widths between
those of its other tests."""
import pytest
import torch

import paper_2508_07329_amd as haq
from tests import fp8_reference as ref
from tests.fp8_sizes import HALVES, ROWS16, STREAM, TILED
from tests.test_fp8 import check_norm

DEV = "cuda:0"
F16, BF16 = torch.float16, torch.bfloat16
MORE = [(33, 1168, 5008), (33, 2064, 4176), (33, 1040, 5424),  # streaming, 16 rows x 64 channels in several tiles of rows
        (65, 16, 4176), (65, 1040, 5008), (80, 2144, 4384), (129, 1040, 2928),  # 32 x 64 in several tiles
        (33, 16, 5632), (63, 2144, 7712), (64, 1040, 6672)]  # 64 x 32 in one
PACKED = [size for shapes in (STREAM, TILED) for sizes in shapes.values() for size in sizes] + HALVES + MORE
FEW = [size for sizes in ROWS16.values() for size in sizes]


def problem(T, K, N, dtype):
    """(rows, packed weights, their scales, y in 64 bits, bound of the sum's error)."""
    x = ref.rows(T * K + N, T, K, dtype)
    w = torch.randn(K, N, generator=torch.Generator().manual_seed(T + K + N)) * 0.02
    wq, sw = ref.weight_codes(w)
    want, bound = ref.linear(*ref.act_codes(x.float()), wq, sw)
    return x.to(DEV), ref.pack_weight(wq).to(DEV), sw.to(DEV), want, bound


def check(y, want, bound, act):
    """(ReLU brings no two numbers further apart.)"""
    ref.assert_linear(y.cpu(), want.clamp(min=0) if act == haq.HAQ_ACT_RELU else want, bound)
    assert act == haq.HAQ_ACT_NONE or bool((y >= 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("T,K,N", PACKED)
def test_on_codes(T, K, N):
    x, wp, sw, want, bound = problem(T, K, N, F16)
    q, s = haq.haq_quant_act_fp8_packed(x)
    for dtype, act in ((F16, haq.HAQ_ACT_NONE), (F16, haq.HAQ_ACT_RELU), (BF16, haq.HAQ_ACT_RELU)):
        wide = torch.full((T + 1, N + 8), 7.0, dtype=dtype, device=DEV)
        haq.haq_gemm_fp8_packed(q, s, wp, sw, T, K, N, act, out=wide[:T, :N])
        check(wide[:T, :N], want, bound, act)
        assert bool((wide[:T, N:] == 7.0).all()) and bool((wide[T] == 7.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("T,K,N", FEW)
def test_on_few_rows(T, K, N):
    for dtype, act in ((F16, haq.HAQ_ACT_NONE), (F16, haq.HAQ_ACT_RELU), (BF16, haq.HAQ_ACT_RELU)):
        x, wp, sw, want, bound = problem(T, K, N, dtype)
        wide = torch.full((T + 1, N + 8), 7.0, dtype=dtype, device=DEV)
        haq.haq_fp8_linear(x, wp, sw, N, act, out=wide[:T, :N])
        check(wide[:T, :N], want, bound, act)
        assert bool((wide[:T, N:] == 7.0).all()) and bool((wide[T] == 7.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("T,K", [(520, 5008), (1500, 8192), (2049, 4096), (2050, 2320)])
@pytest.mark.parametrize("codes", [haq.HAQ_CODES_I8, haq.HAQ_CODES_E4M3])
def test_norm_between(T, K, codes):
    weight = 1.0 + 0.2 * torch.randn(K, generator=torch.Generator().manual_seed(K))
    for dtype in (F16, BF16):
        x, r = ref.rows(T + K, T, K, dtype), ref.rows(T + K + 1, T, K, dtype)
        check_norm(x, weight, r, codes, dtype == F16)
    check_norm(x, weight, None, codes, False)
