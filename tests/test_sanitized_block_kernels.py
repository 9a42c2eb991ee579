"""The kernels of a trained block, compiled for the host (tests/hip_cpu_shim: a lane is a fibre, matrix instructions and exchanges
between lanes are made of their definitions, copies to LDS arrive when they are waited for and no earlier), under AddressSanitizer and
UBSan (CPU only).  Every matrix is a heap block of its size, every array in LDS one of its own; what comes out is compared with the
formulas in 64 bits."""
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
    out = tmp_path_factory.mktemp("block_shim")
    res = subprocess.run([os.path.join(ROOT, "tests", "hip_cpu_shim", "build_block.sh"), CSRC, str(out)], capture_output=True, text=True,
                         env=dict(os.environ, SHIM_CXX=cxx), timeout=900)
    assert res.returncode == 0, res.stdout + res.stderr

    env = dict(ENV, ASAN_OPTIONS=ENV["ASAN_OPTIONS"] + ":detect_stack_use_after_return=0")       # (a second stack for every lane)

    def run(*args):
        res = subprocess.run([str(out / "block_driver")] + [str(v) for v in args], capture_output=True, text=True, env=env, timeout=600)
        assert res.returncode == 0, res.stdout + res.stderr
        assert " values" in res.stdout
    return run


@pytest.mark.parametrize("mode", [F32, BF16, F16])
@pytest.mark.parametrize("columns,p,ld,residual,tokens", [(1, 0.5, 0, 0, [1]), (37, 0.3, 0, 1, [3, 0, 4]), (64, 1.0, 71, 0, [5]),
                                                          (2049, 0.1, 2051, 1, [0, 2])])
def test_dropout(driver, mode, columns, p, ld, residual, tokens):
    driver("dropout", mode, columns, p, ld, residual, *tokens)


# widths of every number of wavefronts and packs that hold a row; a chunk and more, files of none
@pytest.mark.parametrize("mode,centred", [(F32, 0), (F32, 1), (BF16, 1), (F16, 0)])
@pytest.mark.parametrize("width,gate,parts,ld,tokens", [
    (1, 0, "fnr", 0, [2]), (100, 1, "fnr", 0, [3, 0, 35]), (512, 2, "fn", 515, [9, 1]), (700, 2, "fr", 703, [5, 0, 2]),
    (1024, 1, "nr", 0, [3]), (1501, 1, "fnr", 0, [5]), (3000, 2, "fnr", 3001, [2, 1]), (5003, 0, "fnr", 0, [2]), (9001, 1, "fnr", 0, [2])])
def test_joins(driver, mode, centred, width, gate, parts, ld, tokens):
    driver("join", mode, centred, width, 0.2, ld, gate, parts, *tokens)


@pytest.mark.parametrize("mode", [F32, BF16, F16])
@pytest.mark.parametrize("rows,width,hidden,ld", [(1, 1, 1, 0), (1, 264, 72, 0), (4, 51, 133, 53), (7, 130, 40, 0), (16, 51, 133, 0), (27, 72, 101, 79),
                                                  (61, 140, 50, 0)])
def test_few_rows(driver, mode, rows, width, hidden, ld):
    """The kernels that take the weights from memory to the matrix instructions; fewer rows than the batch has."""
    driver("ffn", mode, 0, width, hidden, 0.25, ld, 0, rows, -1, rows // 2, 0, rows - rows // 2 + 3)


# tiles: 1 large, 2 small, 0 small with more of a tile on its way
@pytest.mark.parametrize("mode,tile", [(F32, 0), (F32, 1), (BF16, 0), (BF16, 1), (BF16, 2), (F16, 1)])
@pytest.mark.parametrize("width,hidden,p,ld,tokens", [(8, 8, 0, 0, [1]), (51, 133, 0.3, 60, [20, 0, 21])])
def test_training(driver, mode, tile, width, hidden, p, ld, tokens):
    driver("ffn", mode, 1, width, hidden, p, ld, 1, 0, tile, *tokens)


@pytest.mark.parametrize("mode,tile", [(F32, 0), (BF16, 0), (BF16, 1)])
@pytest.mark.parametrize("width,hidden,tokens", [(330, 24, [0, 5]), (24, 330, [3]), (16, 24, [330, 0])])
def test_training_in_many_steps(driver, mode, tile, width, hidden, tokens):
    """Six steps of 64 in the first product, in those over the hidden values, in the weights' gradients."""
    driver("ffn", mode, 2, width, hidden, 0.1, 0, 1, 0, tile, *tokens)


@pytest.mark.parametrize("mode", [F32, BF16])
@pytest.mark.parametrize("rows,width,hidden,ld", [(66, 40, 1100, 45), (70, 9, 1030, 0)])
def test_second_product_in_ranges(driver, mode, rows, width, hidden, ld):
    driver("ffn", mode, 2, width, hidden, 0.1, ld, 0, rows, -1, rows + 5)


@pytest.mark.parametrize("mode,tile,hidden,rows", [(F32, 0, 40, 140), (F16, 2, 72, 150), (BF16, 1, 72, 260)])
def test_rows_of_more_than_one_tile(driver, mode, tile, hidden, rows):
    """In 16 bits with matrices that the products take as they are: what a tile has past the last row or column is past their ends."""
    driver("ffn", mode, 0, 136, hidden, 0.1, 0, 1, 0, tile, rows, 1)
