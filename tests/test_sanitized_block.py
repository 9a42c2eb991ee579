"""The host side of a trained block under AddressSanitizer and UBSan (CPU only)."""
import os
import subprocess
from fractions import Fraction

import pytest

from test_sanitized_host_code import CSRC, ENV, ROOT, SAN


@pytest.fixture(scope="module")
def sweep(tmp_path_factory):
    out = tmp_path_factory.mktemp("block")
    objs = []
    for src in (os.path.join(CSRC, "block.cpp"), os.path.join(ROOT, "tests", "sanitize", "block_sweep.cpp")):
        objs.append(str(out / (os.path.basename(src) + ".o")))
        subprocess.run(["g++", "-std=c++17"] + SAN + ["-Wall", "-Wextra", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", src,
                                                      "-o", objs[-1]], check=True)
    exe = str(out / "block_sweep")
    subprocess.run(["g++"] + SAN + objs + ["-o", exe], check=True)

    def run(*args):
        res = subprocess.run([exe] + [str(a) for a in args], capture_output=True, text=True, env=ENV, timeout=300)
        assert res.returncode == 0, res.stdout + res.stderr
        return res.stdout
    return run


def test_thresholds_of_dropout_go_to_the_nearest_even(sweep):
    """ccdc.h: rint(65536 p), in exact arithmetic here; ties at both parities, and the doubles beside them."""
    ps = [0.0, 0.1, 0.3, 0.5, 0.9999, 1.0, 1e-9, 2.0 ** -17 * (1 + 2.0 ** -52), 1 - 2.0 ** -18]
    for k in (0, 1, 2, 3, 6552, 6553, 32767, 65534, 65535):
        tie = (k + 0.5) / 65536
        ps += [tie, tie * (1 - 2.0 ** -52), tie * (1 + 2.0 ** -52)]
    got = [int(v) for v in sweep("thresholds", *(p.hex() for p in ps)).split()]
    assert got == [round(Fraction(p) * 65536) for p in ps]


@pytest.mark.parametrize("rows", [0, 1, 31, 32, 33, 4096, (1 << 31) - 33, (1 << 31) - 32, (1 << 31) - 31, (1 << 31) - 1])
def test_chunks_of_files_up_to_the_longest(sweep, rows):
    """Up to the 2^31-1 tokens that a batch may have, where the row after the last chunk is no 32-bit number."""
    assert int(sweep("chunks", rows)) == -(-rows // 32)


def test_tables_and_regions_of_batches(sweep):
    """csrc/block.cpp over configurations and batches: its tables, and that what is saved and the workspace hold what the calls index."""
    assert int(sweep("batches").removeprefix("clean: ")) == 4 * 12 * 7 * 10
