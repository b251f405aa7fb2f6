"""Rows with infinities and NaN through the norm's int8 codes and the int8 product: NaN, or zero behind its ReLU, in their own rows alone."""
import pytest
import torch

import paper_2508_07329_amd as haq
from tests import fp8_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("T", [4, 40, 300, 2100])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_rows_that_are_not_finite(T, dtype):
    K, N = 272, 400
    x = ref.rows(T, T, K, dtype)
    x[1, 3], x[3, 270] = float("inf"), float("nan")
    w = (torch.randn(K, N, generator=torch.Generator().manual_seed(1)) * 0.02).to(DEV)
    wq, sw = haq.haq_quant_weight(w, None)
    _, _, q, s = haq.haq_rmsnorm_quant(x.to(DEV), torch.ones(K, device=DEV), 1e-5, haq.HAQ_CODES_I8)
    bad = torch.tensor([1, 3])
    fine = torch.tensor([i for i in range(T) if i not in (1, 3)])
    want_q, want_s = ref.i8_codes(ref.norm(x, torch.ones(K), 1e-5)[1][fine])
    want = (want_q.double() @ wq.cpu().double()) * want_s.double()[:, None] * sw.cpu().double()
    for act in (haq.HAQ_ACT_NONE, haq.HAQ_ACT_RELU):
        y = haq.haq_gemm_w8a8_packed(q, s, haq.haq_pack_weight(wq), sw, T, K, N, act).cpu()
        assert bool(y[bad].isnan().all() if act == haq.HAQ_ACT_NONE else (y[bad] == 0).all())
        # three roundings of binary32 and one of binary16 (of half the smallest step where it is subnormal)
        w_ = want.clamp(min=0) if act == haq.HAQ_ACT_RELU else want
        assert bool(((y[fine].double() - w_).abs() <= w_.abs() * (2.0 ** -11 + 2.0 ** -22) + 2.0 ** -25).all())
