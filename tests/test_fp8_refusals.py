"""What the 8-bit floating-point calls and the norm refuse, on the host and before any HIP call; runs without a GPU."""
import ctypes as C
import math

import pytest
import torch

import paper_2508_07329_amd as haq
from paper_2508_07329_amd import binding

ONE, ODD = 16, 24  # addresses that are never dereferenced; ODD is not 16-byte aligned
BAD_ARG, UNSUPPORTED, WORKSPACE = -1, -2, -3


ORDER = {
    "haq_quant_weight_fp8": dict(w=ONE, K=256, N=64, wq=ONE, w_scale=ONE, stream=None),
    "haq_quant_act_fp8_packed": dict(x=ONE, ldx=256, dtype=0, T=4, K=256, q=ONE, scale=ONE, stream=None),
    "haq_gemm_fp8_packed": dict(q=ONE, scale=ONE, w=ONE, w_scale=ONE, T=4, K=256, N=64, act=0, dtype=0, y=ONE, ldy=64, stream=None),
    "haq_fp8_linear": dict(x=ONE, ldx=256, dtype=0, w=ONE, w_scale=ONE, T=4, K=256, N=64, act=0, y=ONE, ldy=64, workspace=256, bytes=0, stream=None),
    "haq_rmsnorm_quant": dict(x=ONE, ldx=256, residual=ONE, ldr=256, weight=ONE, eps=1e-5, dtype=0, T=4, K=256, sum=ONE, lds=256, y=ONE,
                              ldy=256, codes=1, q=ONE, scale=ONE, stream=None),
}
POINTERS = ("x", "residual", "weight", "sum", "y", "q", "scale", "w", "wq", "w_scale", "workspace")


def call(name, **changes):
    """The entry point on arguments that are in order but for `changes`."""
    assert set(changes) <= set(ORDER[name])
    return getattr(haq.lib(), name)(*{**ORDER[name], **changes}.values())


COMMON = [("dtype", 2, UNSUPPORTED), ("dtype", -1, UNSUPPORTED), ("T", -1, BAD_ARG), ("T", (1 << 24) + 1, UNSUPPORTED), ("K", 0, BAD_ARG), ("K", 264, UNSUPPORTED),
          ("K", 65552, UNSUPPORTED)]


@pytest.mark.parametrize("name,arg,value,code", [
    *[("haq_quant_act_fp8_packed", *c) for c in COMMON], *[("haq_gemm_fp8_packed", *c) for c in COMMON], *[("haq_fp8_linear", *c) for c in COMMON],
    *[("haq_rmsnorm_quant", *c) for c in COMMON],
    *[("haq_quant_act_fp8_packed", a, v, BAD_ARG) for a in ("x", "q", "scale") for v in (None, ODD)],
    *[("haq_quant_act_fp8_packed", "ldx", v, BAD_ARG) for v in (248, 257, 260, -256)],
    *[("haq_gemm_fp8_packed", a, v, BAD_ARG) for a in ("q", "scale", "w", "w_scale", "y") for v in (None, ODD)],
    *[("haq_gemm_fp8_packed", "ldy", v, BAD_ARG) for v in (56, 65, 68)],
    *[(n, "N", v, c) for n in ("haq_gemm_fp8_packed", "haq_fp8_linear", "haq_quant_weight_fp8") for v, c in ((0, BAD_ARG), (40, UNSUPPORTED), ((1 << 24) + 16, UNSUPPORTED))],
    *[(n, "act", 2, UNSUPPORTED) for n in ("haq_gemm_fp8_packed", "haq_fp8_linear")],
    *[("haq_fp8_linear", a, v, BAD_ARG) for a in ("x", "w", "w_scale", "y") for v in (None, ODD)],
    ("haq_fp8_linear", "ldx", 248, BAD_ARG), ("haq_fp8_linear", "ldy", 68, BAD_ARG),
    ("haq_fp8_linear", "workspace", None, WORKSPACE), ("haq_fp8_linear", "bytes", 4096, WORKSPACE),
    *[("haq_quant_weight_fp8", a, v, BAD_ARG) for a in ("w", "wq", "w_scale") for v in (None, ODD)],
    ("haq_quant_weight_fp8", "K", 24, UNSUPPORTED), ("haq_quant_weight_fp8", "K", -16, BAD_ARG),
    *[("haq_rmsnorm_quant", a, ODD, BAD_ARG) for a in ("x", "residual", "weight", "sum", "y", "q", "scale")],
    *[("haq_rmsnorm_quant", a, None, BAD_ARG) for a in ("x", "weight", "q", "scale", "residual")],  # (a sum without a residual)
    *[("haq_rmsnorm_quant", a, v, BAD_ARG) for a in ("ldx", "ldr", "lds", "ldy") for v in (240, 260)],
    *[("haq_rmsnorm_quant", "eps", v, BAD_ARG) for v in (0.0, -1e-5, math.nan, math.inf, 1e-31)],
    ("haq_rmsnorm_quant", "codes", 3, UNSUPPORTED), ("haq_rmsnorm_quant", "codes", 0, BAD_ARG),
])
def test_refused(name, arg, value, code):
    assert call(name, **{arg: value}) == code
    assert haq.lib().haq_last_error().decode().startswith(name + ":")


@pytest.mark.parametrize("name", ["haq_gemm_fp8_packed", "haq_fp8_linear"])
def test_more_outputs_than_a_launch_reaches_are_refused(name):
    assert call(name, T=1 << 23, N=(1 << 15) + 16, ldy=1 << 16) == UNSUPPORTED
    assert "2^38" in haq.lib().haq_last_error().decode()


def test_norm_without_any_output_is_refused():
    assert call("haq_rmsnorm_quant", codes=0, q=None, scale=None, y=None) == BAD_ARG


@pytest.mark.parametrize("buffers", [dict(q_packed=torch.zeros(16)), dict(scale=torch.zeros(4))])
def test_norm_with_buffers_for_codes_that_it_is_not_asked_for_is_refused(buffers):
    with pytest.raises(haq.HaqError, match="codes"):
        binding.haq_rmsnorm_quant(torch.zeros(4, 256, dtype=torch.float16), torch.ones(256), 1e-5, **buffers)


@pytest.mark.parametrize("name", ["haq_quant_act_fp8_packed", "haq_gemm_fp8_packed", "haq_fp8_linear", "haq_rmsnorm_quant"])
def test_no_tokens_need_no_buffers(name):
    assert call(name, T=0, **{k: None for k in ORDER[name] if k in POINTERS}) == 0


def test_argument_types_of_the_norm_are_those_of_the_header():
    import re
    from tests.test_abi_cpu import _header
    params = re.search(r"\bint32_t\s+haq_rmsnorm_quant\s*\(([^)]*)\)", _header()).group(1).split(",")
    of = lambda p: C.c_void_p if "*" in p else {"int32_t": C.c_int32, "int64_t": C.c_int64, "double": C.c_double}[p.split()[-2]]
    assert list(binding._NORM_TYPES) == [of(p) for p in params]


def test_sizes():
    assert haq.haq_act_scales_fp8_bytes(1, 16) == 4 * 272 and haq.haq_act_scales_fp8_bytes(17, 257) == 4 * 3 * 288
    assert haq.haq_act_scales_fp8_bytes(-1, 16) == 0 and haq.haq_fp8_linear_workspace_bytes(4, 0, 16) == 0
    for T, K in ((1, 16), (33, 2064), (4096, 14336)):
        assert haq.haq_fp8_linear_workspace_bytes(T, K, 64) >= haq.haq_packed_act_bytes(T, K) + haq.haq_act_scales_fp8_bytes(T, K)


@pytest.mark.parametrize("what,says", [("type", "fp16 or bf16"), ("other type", "like the others"), ("shape", "like the others"),
                                       ("strides", "next to each other"), ("device", "current GPU")])
def test_rows_that_the_binding_refuses(what, says):
    x, r, w = torch.zeros(4, 32, dtype=torch.float16), torch.zeros(4, 32, dtype=torch.float16), torch.ones(32)
    if what == "type":
        x = x.float()
    if what == "other type":
        x, r = r, x.bfloat16()
    if what == "shape":
        x, r = r, x[:3]
    if what == "strides":
        x = torch.zeros(32, 4, dtype=torch.float16).t()
    tensors = {"x": x} if what in ("type", "strides") else {"x": x, "residual": r}
    with pytest.raises(haq.HaqError, match="current GPU" if what in ("other type", "shape") else says):
        haq.haq_rmsnorm_quant(x, w, 1e-5, residual=r)
    if what in ("other type", "shape"):  # the rows themselves, without a look at where they are
        import unittest.mock as mock
        with mock.patch.object(binding, "_here", lambda *a: None), pytest.raises(haq.HaqError, match=says):
            binding._rows16("haq_rmsnorm_quant", **tensors)


def test_buffers_that_the_binding_refuses(monkeypatch):
    monkeypatch.setattr(binding, "_here", lambda *a: None)
    flat = lambda t, dt, n: binding._flat("call", "buffer", t, dt, n)
    flat(torch.zeros(4), torch.float32, 4)
    for t in (torch.zeros(3), torch.zeros(4, dtype=torch.float16), torch.zeros(4, 2)[:, 0]):
        with pytest.raises(haq.HaqError, match="buffer must be a contiguous"):
            flat(t, torch.float32, 4)
    with pytest.raises(haq.HaqError, match="haq_pack_weight"):
        binding._fp8_weights("call", torch.zeros(128 * 256 - 1, dtype=torch.int8), torch.zeros(1), 128, 16)
