"""The kernels that learn from a teacher compiled for the host (tests/hip_cpu_shim: lanes as fibres, the instructions that cross lanes
made of their definitions, copies to LDS arrive when they are waited for and no earlier), under AddressSanitizer and UBSan (CPU
only).  Every matrix is a heap block of its size, every array in LDS one of its own; what comes out is compared with the formulas in 64
bits."""
import os
import shutil
import subprocess

import pytest

from test_sanitized_host_code import CSRC, ENV, ROOT

F32, BF16, F16 = 0, 3, 4          # enum ccdc_mode


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    cxx = "/opt/rocm/lib/llvm/bin/clang++"
    if not os.path.exists(cxx):
        cxx = shutil.which("clang++")
    if not cxx:
        pytest.skip("no clang++ to build the kernels for the host")
    out = tmp_path_factory.mktemp("teacher_shim")
    res = subprocess.run([os.path.join(ROOT, "tests", "hip_cpu_shim", "build_teacher.sh"), CSRC, str(out)], capture_output=True, text=True,
                         env=dict(os.environ, SHIM_CXX=cxx), timeout=900)
    assert res.returncode == 0, res.stdout + res.stderr

    env = dict(ENV, ASAN_OPTIONS=ENV["ASAN_OPTIONS"] + ":detect_stack_use_after_return=0")       # (a second stack for every lane)

    def run(*args):
        res = subprocess.run([str(out / "teacher_driver")] + [str(v) for v in args], capture_output=True, text=True, env=env, timeout=600)
        assert res.returncode == 0, res.stdout + res.stderr
        assert " values" in res.stdout
    return run


@pytest.mark.parametrize("mode", [F32, BF16, F16])
@pytest.mark.parametrize("rows,columns,pad", [(1, 1, 0), (3, 127, 1), (2, 129, 0), (5, 300, 3), (1, 640, 0)])
def test_quantise(driver, mode, rows, columns, pad):
    driver("quantise", mode, rows, columns, pad)


# kernels for few rows: every one of them, parts of k that end before others, groups past the last row of the weights
@pytest.mark.parametrize("mode", [F32, BF16, F16])
@pytest.mark.parametrize("rows,wide,outputs,pad", [(1, 1024, 3, 0), (4, 1152, 21, 1), (5, 1152, 9, 0), (8, 1664, 33, 2), (11, 1024, 17, 0), (16, 1152, 20, 0), (25, 1152, 18, 3),
                                                   (50, 1024, 19, 0)])
def test_products_of_few_rows(driver, mode, rows, wide, outputs, pad):
    driver("product", mode, rows, wide, outputs, pad, -1)


@pytest.mark.parametrize("mode,rows,outputs", [(F16, 3, 8195), (F32, 10, 8200), (BF16, 18, 8193)])
def test_products_of_few_rows_and_many_outputs(driver, mode, rows, outputs):
    driver("product", mode, rows, 1024, outputs, 0, -1) if mode == F16 else driver("product", F32, rows, 1024, outputs, 0, -1)


# tiles: 1 largest, 2 of 64 x 64, 3 of 64 x 128, 4 of 128 x 128 with more of it in LDS, 5 of 128 x 128
@pytest.mark.parametrize("mode,tile", [(BF16, 1), (BF16, 2), (BF16, 3), (F16, 4), (F16, 5), (F32, 2), (F32, 3), (F32, 4), (F32, 5)])
@pytest.mark.parametrize("rows,wide,outputs,pad", [(1, 128, 1, 0), (70, 256, 130, 3), (9, 1152, 20, 0), (133, 640, 67, 0)])
def test_products_by_tiles(driver, mode, tile, rows, wide, outputs, pad):
    driver("product", mode, rows, wide, outputs, pad, tile)


def test_products_of_more_than_one_tile(driver):
    driver("product", BF16, 260, 256, 270, 1, 1)
    driver("product", F16, 140, 128, 270, 0, 5)


# rows by every number of wavefronts, held and read again; few rows and many
@pytest.mark.parametrize("mode,kind", [(F32, 0), (BF16, 1), (F16, 2), (BF16, 0)])
@pytest.mark.parametrize("rows,columns,k,pad", [(2, 1, 3, 0), (1, 7, 2, 1), (3, 130, 128, 0), (2, 700, 20, 1), (258, 1500, 5, 0), (1, 4001, 9, 0), (257, 2500, 3, 0),
                                                (1, 8100, 30, 3)])
def test_top(driver, mode, kind, rows, columns, k, pad):
    driver("top", mode, rows, columns, k, pad, kind)


@pytest.mark.parametrize("mode,columns", [(BF16, 16000), (F32, 33000), (F16, 66001), (F32, 66001), (BF16, 132000)])
def test_top_of_long_rows(driver, mode, columns):
    driver("top", mode, 1, columns, 17, 0, 0)


def test_top_of_more_equal_logits_than_the_list_has_room_for(driver):
    for columns in (300, 3000, 20000):
        driver("top", BF16, 1, columns, 20, 0, 1)


@pytest.mark.parametrize("mode,place", [(F32, 0), (F32, 1), (BF16, 0), (F16, 1)])
@pytest.mark.parametrize("rows,columns,k,pad", [(2, 41, 3, 0), (5, 130, 128, 1), (4, 700, 20, 0), (258, 1100, 5, 0), (1, 4001, 9, 3), (257, 2500, 3, 0), (2, 8100, 30, 0)])
def test_distill(driver, mode, place, rows, columns, k, pad):
    driver("distill", mode, rows, columns, k, pad, place)


@pytest.mark.parametrize("mode,columns", [(BF16, 16000), (F32, 32000), (F16, 33001), (F32, 60001), (BF16, 66001), (F32, 66001)])
def test_distill_of_long_rows(driver, mode, columns):
    driver("distill", mode, 2, columns, 40, 1, 0)
