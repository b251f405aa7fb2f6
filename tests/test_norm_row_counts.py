"""A row of the norm gives the same bits whatever the number of rows around it, hence whatever kernel takes it."""
import math
from fractions import Fraction

import pytest
import torch

import paper_2508_07329_amd as haq
from tests import fp8_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def border_eps(row):
    """An eps for which 1 / sqrt(mean of squares + eps) lies on the border between two values of binary32, and the mean: there the
    rounded root shows the last bit of the binary64 sum."""
    m = sum(Fraction(v) ** 2 for v in row.double().tolist()) / row.numel()
    inv = torch.tensor(1.0 / math.sqrt(float(m) + 1e-5), dtype=torch.float32)
    below = torch.nextafter(inv, torch.tensor(0.0))
    border = (Fraction(inv.item()) + Fraction(below.item())) / 2
    return float(1 / border ** 2 - m), float(m)


@pytest.mark.parametrize("K", [272, 2064, 4096, 8208, 16384])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("codes", [haq.HAQ_CODES_I8, haq.HAQ_CODES_E4M3])
def test_a_row_alone_and_among_others(K, dtype, codes):
    weight = (1.0 + 0.2 * torch.randn(K, generator=torch.Generator().manual_seed(K))).to(DEV)
    for seed in range(4):
        row = ref.rows(seed, 1, K, dtype)
        eps0, m = border_eps(row[0])
        step = math.ulp(m) / 2
        batches = {T: row.to(DEV).expand(T, K).contiguous() for T in (1, 600, 2100)}
        for i in range(-24, 25):
            eps = eps0 + i * step
            assert eps > 0
            alone = None
            for T, x in batches.items():
                y, _, q, s = haq.haq_rmsnorm_quant(x, weight, eps, codes, y=torch.empty_like(x))
                s = s[None, :T] if codes == haq.HAQ_CODES_I8 else s.view(-1, ref.padded_rows(T))[:, :T]
                q = q.view(torch.uint8).view(-1, ref.padded_rows(T), 16)[: K // 16, :T]
                got = (y, s.t(), q.transpose(0, 1))
                alone = alone or tuple(v[:1].clone() for v in got)
                for what, a, b in zip(("rows", "scales", "codes"), got, alone):
                    assert bool((a == b).all()), (what, T, seed, i, eps)
