"""Weights and scales of another layer are refused by the 8-bit floating-point calls and the norm, larger ones as well as smaller: the library
would read them with this layer's strides.  Buffers for codes may be larger.  The library and the GPU are stood in for; runs without one."""
import pytest
import torch

import paper_2508_07329_amd as haq
from paper_2508_07329_amd import binding
from tests.fp8_reference import padded_rows
from tests.test_binding_types import Library

T, K, N = 4, 400, 272
KB, NB = 4, 3  # blocks of 128
F16, E4M3 = torch.float16, torch.float8_e4m3fn


class OnGpu(torch.Tensor):
    def get_device(self):
        return 0


def on_gpu(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


@pytest.fixture
def library(monkeypatch):
    stand_in = Library()
    monkeypatch.setattr(binding, "lib", lambda: stand_in)
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    monkeypatch.setattr(binding, "_raw_stream", lambda dev: 0)
    monkeypatch.setattr(binding, "_here", lambda *a: None)
    return stand_in


def arguments():
    x, out, R = on_gpu(T, K, dtype=F16), on_gpu(T, N, dtype=F16), padded_rows(T)
    w_packed, w_scale = on_gpu(448 * 512, dtype=torch.int8), on_gpu(KB, NB)
    codes, scales = on_gpu(448 * R, dtype=E4M3), on_gpu(KB * R)
    return {
        "haq_quant_weight_fp8": dict(w=on_gpu(K, N), wq=on_gpu(K, N, dtype=E4M3), w_scale=w_scale),
        "haq_quant_act_fp8_packed": dict(x=x, q_packed=codes, block_scale=scales),
        "haq_gemm_fp8_packed": dict(q_packed=codes, block_scale=scales, w_packed=w_packed, w_scale=w_scale, T=T, K=K, N=N, out=out),
        "haq_fp8_linear": dict(x=x, w_packed=w_packed, w_scale=w_scale, N=N, out=out, workspace=on_gpu(1 << 20, dtype=torch.uint8)),
        "haq_rmsnorm_quant": dict(x=x, weight=on_gpu(K), eps=1e-5, codes=haq.HAQ_CODES_E4M3, q_packed=codes, scale=scales),
    }


@pytest.mark.parametrize("name", list(arguments()))
def test_what_fits_passes(library, name):
    getattr(haq, name)(**arguments()[name])
    assert library.calls == [name]


@pytest.mark.parametrize("name,what", [(n, w) for n, a in arguments().items() for w in ("q_packed", "block_scale", "scale") if w in a])
def test_buffers_for_codes_may_be_larger_but_not_smaller(library, name, what):
    args = arguments()[name]
    t = args[what]
    args[what] = on_gpu(t.numel() + 64, dtype=t.dtype)
    getattr(haq, name)(**args)
    assert library.calls == [name]
    args[what] = on_gpu(t.numel() - 1, dtype=t.dtype)
    with pytest.raises(haq.HaqError, match=name):
        getattr(haq, name)(**args)


@pytest.mark.parametrize("name,what,shapes", [
    ("haq_rmsnorm_quant", "weight", [(2 * K,), (K + 1,), (K - 1,)]),
    ("haq_fp8_linear", "w_scale", [(KB, NB + 1), (KB + 1, NB), (KB, NB - 1)]),
    ("haq_gemm_fp8_packed", "w_scale", [(KB, NB + 1), (KB + 1, NB), (KB, NB - 1)]),
    ("haq_fp8_linear", "w_packed", [(448 * 768,), (512 * 512,), (448 * 256,)]),
    ("haq_gemm_fp8_packed", "w_packed", [(448 * 768,), (512 * 512,), (448 * 256,)]),
    ("haq_quant_weight_fp8", "wq", [(K, 2 * N), (N, K), (K - 16, N)]),
    ("haq_quant_weight_fp8", "w_scale", [(KB, NB + 1), (KB + 1, NB), (KB, NB - 1)]),
])
def test_what_is_of_another_layer_is_refused(library, name, what, shapes):
    for shape in shapes:
        args = arguments()[name]
        args[what] = on_gpu(*shape, dtype=args[what].dtype)
        with pytest.raises(haq.HaqError, match=f"{name}: {what}"):
            getattr(haq, name)(**args)
        assert not library.calls
