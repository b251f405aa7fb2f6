"""Every kernel that is built for the 8-bit floating-point calls and the norm is launched by some call, and by some size of the GPU tests: the
host code over the recording stand-in for the HIP runtime."""
import os
import random
import re
import subprocess

import pytest

from paper_2508_07329_amd import build as hip_build
from tests.test_launch_plan import HERE, _host_program


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    sources = [os.path.join(hip_build.CSRC, s) for s in ("fp8_api.hip", "fp8_quant.hip", "fp8_gemm.hip", "fp8_stream.hip", "rmsnorm.hip")]
    return _host_program(tmp_path_factory.mktemp("reached"), "fp8", sources + [os.path.join(HERE, "fp8_launch_recorder.cpp")])


def _kernel(symbol):
    """Name and template arguments but the type of the rows, which the sizes' rules do not look at (the recorder's calls take one)."""
    name = re.search(r"(fp8_gemm_halves|fp8_gemm|fp8_stream|act_quant|weight_quant|rmsnorm)_kernel", symbol).group(1)
    return (name, *[int(v) for v in re.findall(r"L[ib](\d+)E", symbol)][1:])


def built(program):
    symbols = subprocess.run(["nm", program], stdout=subprocess.PIPE, text=True, check=True).stdout
    return {_kernel(line.split()[-1]) for line in symbols.splitlines() if "_kernel" in line and "__device_stub__" not in line}


def launched(program, calls):
    text = "".join(" ".join(map(str, c)) + "\n" for c in calls)
    lines = subprocess.run([program], input=text, stdout=subprocess.PIPE, text=True, check=True).stdout.splitlines()
    assert [line for line in lines if line[0] == "="] == ["= 0"] * len(calls)
    return {_kernel(line.split()[0]) for line in lines if line[0] != "="}


def test_every_kernel_is_launched_by_some_call(program):
    rng = random.Random(1)
    size = lambda most: 16 * int(2 ** rng.uniform(0, most))
    calls = [("w", 128, 128, 0), ("g", 33, 1168, 5008)]
    for _ in range(5000):
        T, K, N = int(2 ** rng.uniform(0, 13)), size(12), size(12)
        calls += [("g", T, K, N), ("l", 1 + T % 8, K, N), ("n", T, K, T % 3), ("q", T, K, 0)]
    kernels = built(program)
    assert len(kernels) > 40
    assert kernels == launched(program, calls)


def test_every_kernel_is_run_by_a_gpu_test(program):
    """In both types: these tests go over the types themselves."""
    from tests import test_fp8, test_fp8_each_kernel
    of = lambda test, names: next(mark.args[1] for mark in test.pytestmark if mark.name == "parametrize" and mark.args[0] == names)
    calls = [("w", *size, 0) for size in of(test_fp8.test_weight_codes, "K,N")]
    calls += [("q", *size, 0) for size in of(test_fp8.test_activation_codes, "T,K")]
    for test in (test_fp8.test_norm, test_fp8_each_kernel.test_norm_between):
        calls += [("n", *size, codes) for size in of(test, "T,K") for codes in of(test, "codes")]
    calls += [("g", *size) for size in of(test_fp8_each_kernel.test_on_codes, "T,K,N")]
    calls += [("l", *size) for size in of(test_fp8_each_kernel.test_on_few_rows, "T,K,N")]
    assert built(program) == launched(program, calls)
