"""The 8-bit floating-point linear where the product of a token's and of a weight block's scale is a subnormal of binary32, or zero."""
import pytest
import torch

import paper_2508_07329_amd as haq
from tests import fp8_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("T,K,N", [(1, 400, 272), (8, 2064, 272), (20, 1040, 272), (60, 2144, 7712), (200, 656, 528), (129, 592, 12432)])
def test_small_scales(T, K, N):
    """Magnitudes whose product goes from 2^-95 to 2^-150: the error that the definition allows, and in binary32 arithmetic 2^-150 for the
    product of the scales (half of the smallest step) of each block, times p_b, and 2^-150 for each sum."""
    rows = ref.rows(T + K, T, K, torch.float32, outliers=False) * 2.0 ** (-45.0 - 55.0 * torch.arange(T) / T)[:, None]
    if T == 1:
        rows *= 2.0 ** -20
    x = rows.bfloat16()
    w = torch.randn(K, N, generator=torch.Generator().manual_seed(N)) * 2.0 ** -54
    (xq, sx), (wq, sw) = ref.act_codes(x.float()), ref.weight_codes(w)
    product = sx.double().amax(dim=1) * sw.double().max()
    assert (product < 2.0 ** -126).any() and (T == 1 or (product > 2.0 ** -126).any())
    want, bound = ref.linear(xq, sx, wq, sw)
    bound = bound + 2.0 ** -150 * (xq.double().abs() @ wq.double().abs() + -(-K // 128))
    y = haq.haq_fp8_linear(x.to(DEV), ref.pack_weight(wq).to(DEV), sw.to(DEV), N)
    ref.assert_linear(y.cpu(), want, bound)
    normal = product > 2.0 ** -120  # where nothing is lost, outputs are not all zero
    assert not bool(normal.any()) or bool((y.cpu()[normal] != 0).any(dim=1).all())
