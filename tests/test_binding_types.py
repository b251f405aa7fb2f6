"""Calls that read and write binary16 rows refuse rows of another type, bfloat16 rows of the norm among them: as binary16 they would be
other numbers.  The library is stood in for, so that nothing is launched; runs without a GPU."""
import pytest
import torch

import paper_2508_07329_amd as haq
from paper_2508_07329_amd import binding

T, K, N, E = 4, 128, 64, 2
F16, BF16 = torch.float16, torch.bfloat16


class Library:
    """Every entry point returns 0 and is noted."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            return 0
        return call


@pytest.fixture
def library(monkeypatch):
    stand_in = Library()
    monkeypatch.setattr(binding, "lib", lambda: stand_in)
    monkeypatch.setattr(binding, "_stream", lambda: None)
    monkeypatch.setattr(binding, "_stream_adr", lambda: 0)
    return stand_in


def arguments():
    f, i = torch.zeros(K), torch.zeros(K * N, dtype=torch.int8)
    expert = haq.ExpertWeights(i, i, f, f, f, f)
    x, logits = torch.zeros(T, K, dtype=F16), torch.zeros(T, E, dtype=F16)
    out, hidden, ws = torch.zeros(T, N, dtype=F16), torch.zeros(T, K, dtype=F16), torch.zeros(256, dtype=torch.uint8)
    wq = torch.zeros(K, N, dtype=torch.int8)
    experts = dict(logits=logits, s_in=f, experts=[expert] * E, I=N, out=hidden)
    return {
        "haq_smooth_quant_act": dict(x=x, s=f),
        "haq_channel_absmax_f16": dict(x=x, ax=f),
        "haq_quant_act_packed": dict(x=x, s=f, q_packed=i, row_scale=f),
        "haq_gemm_w8a8_packed": dict(q_packed=i, row_scale=f, w_packed=i, w_scale=f, T=T, K=K, N=N, out=out),
        "haq_w8a8_linear": dict(x=x, s=f, w_packed=i, w_scale=f, N=N, out=out, workspace=ws),
        "haq_w8a8_linear_kn": dict(x=x, s=f, wq_kn=wq, w_scale=f, out=out, workspace=ws),
        "haq_w8a8_linear_asym": dict(x=x, s=f, w_packed=i, w_scale=f, w_colsum=f, N=N, out=out, workspace=ws),
        "haq_w8a8_ffn": dict(x=x, s1=f, w1_packed=i, w1_scale=f, F=K, act=0, s2=f, w2_packed=i, w2_scale=f, N=N, out=out, workspace=ws),
        "haq_moe_w8a8_ffn": dict(x=x, workspace=ws, **experts),
        "haq_moe_w8a8_ffn_static": dict(x=x, **experts),
        "haq_moe_w8a8_ffn_asym": dict(x=x, colsums=[(f, f, f)] * E, workspace=ws, **experts),
        "haq_cpu_expert_ffn": dict(handle=None, x=x, s_in=f, H=K),
        "haq_reference_matmul_f64": dict(x=x, w=torch.zeros(K, N)),
        "haq_quant_loss_f64": dict(y=out, yref=torch.zeros(T, N, dtype=torch.float64)),
        "haq_smoothing_search": dict(x=x, w=torch.zeros(K, N), exponents=[0.5], workspace=ws),
        "haq_hessian_f64": dict(x=x, s=f),
        "haq_hessian_quant_weight": dict(x=x, w=torch.zeros(K, N), s=f, workspace=ws),
        "haq_quantize_layer": dict(x=x, w=torch.zeros(K, N), exponents=[0.5], workspace=ws),
    }


@pytest.mark.parametrize("name", list(arguments()))
def test_rows_in_binary16_pass(library, name):
    getattr(haq, name)(**arguments()[name])
    assert name in library.calls


@pytest.mark.parametrize("name,what", [(name, what) for name, args in arguments().items() for what in ("x", "y", "logits", "out") if what in args])
@pytest.mark.parametrize("dtype", [BF16, torch.float32])
def test_rows_of_another_type_are_refused(library, name, what, dtype):
    args = arguments()[name]
    args[what] = args[what].to(dtype)
    with pytest.raises(haq.HaqError, match=f"{name}.*fp16.*{str(dtype).split('.')[1]}"):
        getattr(haq, name)(**args)
    assert name not in library.calls


def test_codes_in_8_bit_floating_point_are_no_operand_of_the_int8_product(library):
    args = arguments()["haq_gemm_w8a8_packed"]
    args["q_packed"] = args["q_packed"].view(torch.float8_e4m3fn)
    with pytest.raises(haq.HaqError, match="haq_gemm_w8a8_packed.*int8"):
        haq.haq_gemm_w8a8_packed(**args)
    assert not library.calls
