"""Which kernel a gated product runs (csrc/gemm_rules.h: gated_route) in a host build: no GPU needed."""

import os
import shutil
import subprocess

import pytest

import test_gpu_gated
import test_gpu_ksplit

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def routes(tmp_path_factory):
    """[(of the gated product, of the product alone)] of shapes (M, K, N, bits)."""
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("g++ not available")
    exe = tmp_path_factory.mktemp("rules") / "gated_rules_check"
    r = subprocess.run([gxx, "-O1", "-std=c++17", "-Wall", "-Werror",
                        "-I" + os.path.join(ROOT, "paper_2606_12487_amd", "csrc"),
                        os.path.join(ROOT, "tests", "gated_rules_check.cpp"), "-o", str(exe)],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]

    def ask(shapes):
        run = subprocess.run([str(exe)], input="".join(f"{M} {N} {K} {b}\n" for M, K, N, b in shapes),
                             capture_output=True, text=True, timeout=60)
        assert run.returncode == 0
        return [tuple(line.split()) for line in run.stdout.splitlines()]

    return ask


def test_the_gpu_tests_reach_every_tile(routes):
    assert {r[0] for r in routes(test_gpu_gated.SMALL_CASES)} == {"small"}
    assert {r[0] for r in routes(test_gpu_gated.TALL_CASES)} == {"tall"}
    others = routes(test_gpu_gated.TILE_CASES + test_gpu_ksplit.CASES)
    assert {r[0] for r in others} >= {"decode", "tile", "wide", "ksplit"}


def test_where_the_tiles_are_full_the_kernels_are_those_of_the_product(routes):
    # Few tokens, whole rounds of large tiles, and sizes beyond the fitted ones.
    shapes = [(M, K, N, b) for b in (4, 8) for M, K, N in
              ((1, 4096, 28672), (16, 8192, 57344), (48, 8192, 8192), (512, 4096, 28672), (4001, 8192, 57344),
               (4096, 4096, 22016), (65536, 4096, 22016), (1000000, 8192, 57344), (65536, 65536, 16))]
    assert all(a == b for a, b in routes(shapes)), list(zip(shapes, routes(shapes)))


def test_measured_shapes(routes):
    # 60 -> 44 us, 123 -> 90, 308 -> 243 (256 x 192); 30 -> 22, 11.1 -> 8.1, 36 -> 26 (128 x 128).
    tall = [(333, 4096, 28672, 8), (333, 4096, 28672, 4), (192, 8192, 57344, 8), (570, 8192, 57344, 8)]
    small = [(128, 4096, 28672, 8), (128, 4096, 28672, 4), (300, 1024, 8192, 8), (100, 5120, 27648, 8)]
    assert [r[0] for r in routes(tall + small)] == ["tall"] * 4 + ["small"] * 4
