"""The 8-bit floating-point linear on the longest rows: 65536 channels, and the most whose codes one launch holds for 1, 2, 4 and 8 rows."""
import pytest
import torch

import paper_2508_07329_amd as haq
from tests import fp8_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("T,K,N", [(1, 65536, 48), (1, 65536, 4112), (2, 32768, 80), (4, 16384, 144), (8, 8192, 48), (8, 65536, 48), (40, 65536, 80), (300, 65520, 272),
                                   (70, 65536, 4112)])
def test_linear(T, K, N):
    x = ref.rows(T + K, T, K, torch.float16)
    w = torch.randn(K, N, generator=torch.Generator().manual_seed(N)) * 0.02
    wq, sw = ref.weight_codes(w)
    want, bound = ref.linear(*ref.act_codes(x.float()), wq, sw)
    wp, swd = ref.pack_weight(wq).to(DEV), sw.to(DEV)
    y = haq.haq_fp8_linear(x.to(DEV), wp, swd, N)
    ref.assert_linear(y.cpu(), want, bound)
    q, s = haq.haq_quant_act_fp8_packed(x.to(DEV))
    ref.assert_linear(haq.haq_gemm_fp8_packed(q, s, wp, swd, T, K, N).cpu(), want, bound)
