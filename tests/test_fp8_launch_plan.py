"""Which kernels the 8-bit floating-point calls and the norm launch, and with what grid and LDS: the host code over a recording
stand-in for the HIP runtime."""
import os
import random
import re
import subprocess

import pytest

from paper_2508_07329_amd import build as hip_build
from tests.fp8_sizes import HALVES, ROWS16, STREAM, TILED
from tests.test_launch_plan import HERE, _host_program

MOST_ROWS = 1 << 24


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """plan(calls) -> for each call a list of (kernel, its integer template arguments, (work-groups x, y), threads, LDS bytes)."""
    sources = [os.path.join(hip_build.CSRC, s) for s in ("fp8_api.hip", "fp8_quant.hip", "fp8_gemm.hip", "fp8_stream.hip", "rmsnorm.hip")]
    exe = _host_program(tmp_path_factory.mktemp("fp8"), "fp8", sources + [os.path.join(HERE, "fp8_launch_recorder.cpp")])

    def run(calls):
        text = "".join(" ".join(map(str, c)) + "\n" for c in calls)
        out = subprocess.run([exe], input=text, stdout=subprocess.PIPE, text=True, check=True).stdout
        res, launches = [], []
        for line in out.splitlines():
            if line.startswith("="):
                assert line == "= 0", (calls[len(res)], line)
                res.append(launches)
                launches = []
                continue
            name, gx, gy, threads, lds = line.split()
            kernel = re.search(r"(fp8_gemm_halves|fp8_gemm|fp8_stream|act_quant|weight_quant|rmsnorm)_kernel", name).group(1)
            launches.append((kernel, [int(v) for v in re.findall(r"L[ib](\d+)E", name)], (int(gx), int(gy)), int(threads), int(lds)))
        assert len(res) == len(calls)
        return res

    return run


def cd(a, b):
    return -(-a // b)


def fits_the_machine(launch):
    _, _, (gx, gy), threads, lds = launch
    return gx * threads < 1 << 32 and gy < 1 << 16 and 64 <= threads <= 1024 and lds <= 160 * 1024


def work_groups(kernel, t, M, N, n_cu):
    """What the grid has to reach."""
    if kernel == "fp8_gemm":
        return cd(M, t[1]) * cd(N, t[2])
    if kernel == "fp8_gemm_halves":  # whole rounds of tiles, and at most one of halves; every XCD a share of both
        tiles = cd(M, 256) * cd(N, 256)
        assert tiles > n_cu and 0 < 2 * (tiles % n_cu) <= n_cu
        return cd(tiles - tiles % n_cu, 8) * 8 + cd(2 * (tiles % n_cu), 8) * 8
    assert kernel == "fp8_stream"
    return (cd(M, 16 * t[2]) if t[7] else 1) * cd(N, 16 * t[1])


def test_every_tile_of_a_linear_has_a_work_group(plan):
    rng = random.Random(3)
    sizes = [(int(2 ** rng.uniform(0, 12.5)), 16 * int(2 ** rng.uniform(0, 10)), 16 * int(2 ** rng.uniform(0, 10.5))) for _ in range(1500)]
    sizes += [(M, K, N) for M in (1, 8, 9, 16, 17, 64, 65, 8192) for K in (16, 65536) for N in (16, 65536, MOST_ROWS)]
    sizes += [(MOST_ROWS, 4096, 4096), (MOST_ROWS, 16, 8192), (MOST_ROWS, 65536, 16384), (1 << 19, 16, 1 << 19), (200000, 65536, 16), (100000, 4096, 131072)]
    for n_cu in (256, 64, 304):
        calls = [("c", n_cu, 0, 0)] + [("g", *s) for s in sizes]
        for (M, K, N), launches in zip(sizes, plan(calls)[1:]):
            (kernel, t, grid, threads, lds), = launches
            assert fits_the_machine(launches[0]), (M, K, N, launches)
            assert grid[0] * grid[1] >= work_groups(kernel, t, M, N, n_cu), (M, K, N, launches)
            if kernel == "fp8_gemm_halves":
                assert grid[0] % 8 == 0 and threads == 512 and lds == 2 * (512 * 128 + 8 * 256)
            elif kernel == "fp8_gemm":
                assert grid[0] % 8 == 0 and threads == 64 * t[3] * t[4] * t[6] and lds == t[6] * t[5] * ((t[1] + t[2]) * 128 + t[3] * t[4] * 256)
            else:
                assert t[6] == 0 and (t[7] == 1 or M <= 16 * t[2]) and threads == 64 * t[3] and lds == t[3] * t[1] * t[2] * 1024


def test_sizes_of_the_gpu_tests_take_the_kernels_that_they_are_for(plan):
    for shape, sizes in STREAM.items():
        for s, launches in zip(sizes, plan([("g", *s) for s in sizes])):
            (kernel, t, *_), = launches
            assert kernel == "fp8_stream" and (16 * t[2], 16 * t[1]) == shape, (s, shape, launches)
    for shape, sizes in TILED.items():
        for s, launches in zip(sizes, plan([("g", *s) for s in sizes])):
            (kernel, t, *_), = launches
            assert kernel == "fp8_gemm" and (t[1], t[2], t[6]) == shape, (s, shape, launches)


def test_sizes_of_the_gpu_test_of_few_rows_take_the_kernels_that_they_are_for(plan):
    for (channels, room), sizes in ROWS16.items():
        for s, launches in zip(sizes, plan([("l", *s) for s in sizes])):
            (kernel, t, *_), = launches
            assert kernel == "fp8_stream" and (16 * t[1], t[6]) == (channels, room), (s, launches)


def test_halves_of_the_last_tiles(plan):
    """Where the tiles behind whole rounds fill at most half of one."""
    halves = HALVES + [(4096, 4096, 14336), (2304, 4096, 8192), (4096, 2048, 4352)]
    whole = [(4096, 4096, 4096), (8192, 8192, 8192), (3000, 4096, 14336)]
    of = lambda sizes: {launches[0][0] for launches in plan([("g", *s) for s in sizes])}
    assert of(halves) == {"fp8_gemm_halves"} and of(whole) == {"fp8_gemm"}


def test_a_few_rows_take_one_launch_and_more_two(plan):
    """Rows whose codes fit 64 KB of LDS; the work-groups of the one launch hold them."""
    one = [(1, 16, 16), (1, 65536, 16), (2, 32768, 64), (3, 16384, 64), (4, 16384, 4112), (5, 8192, 8208), (8, 8192, 65536), (8, 1040, 16)]
    two = [(2, 32784, 64), (3, 16400, 64), (5, 8208, 64), (9, 16, 16), (64, 4096, 4096), (300, 64, 64)]
    for s, launches in zip(one, plan([("l", *s) for s in one])):
        (kernel, t, grid, _, lds), = launches
        assert kernel == "fp8_stream" and t[6] >= s[0] and fits_the_machine(launches[0]) and grid[0] == cd(s[2], 16 * t[1]), (s, launches)
        assert lds >= t[3] * t[1] * 1024 + t[6] * cd(s[1], 1024) * 8 * 132, (s, launches)
    for s, launches in zip(two, plan([("l", *s) for s in two])):
        assert [k for k, *_ in launches][0] == "act_quant" and len(launches) == 2, (s, launches)


def test_quantisers_and_norm_cover_every_row_and_channel(plan):
    rng = random.Random(4)
    sizes = [(int(2 ** rng.uniform(0, 14)), 16 * int(2 ** rng.uniform(0, 12))) for _ in range(400)]
    sizes += [(MOST_ROWS, 16), (MOST_ROWS, 8192), (MOST_ROWS, 65536), (MOST_ROWS - 1, 16400), (1, 65536), (7, 16), (8, 16384), (2048, 16384), (2048, 16400)]
    for codes in (0, 1, 2):
        for (T, K), launches in zip(sizes, plan([("n", T, K, codes) for T, K in sizes])):
            (kernel, t, grid, threads, lds), = launches
            assert kernel == "rmsnorm" and fits_the_machine(launches[0]), (T, K, launches)
            rows, pieces = t[1], t[2]
            assert grid[0] * grid[1] * rows >= T and threads // 64 * pieces * (64 // rows) >= cd(K, 16), (T, K, launches)
    for dtype in (0, 1):
        for (T, K), launches in zip(sizes, plan([("q", T, K, dtype) for T, K in sizes])):
            assert len(launches) == 1 and launches[0][0] == "act_quant" and fits_the_machine(launches[0]), (T, K, launches)
    for (K, N), launches in zip([(16, 16), (65536, 16), (16, MOST_ROWS), (65536, 65536)], plan([("w", 16, 16, 0), ("w", 65536, 16, 0), ("w", 16, MOST_ROWS, 0), ("w", 65536, 65536, 0)])):
        assert launches[0][2] == (cd(N, 128), cd(K, 128)) and fits_the_machine(launches[0])
