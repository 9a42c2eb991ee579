"""As test_sanitized_teacher_kernels.py: products whose scales are next to their ends, by every kernel."""
import pytest

from test_sanitized_teacher_kernels import BF16, F16, F32, driver  # noqa: F401


@pytest.mark.parametrize("mode", [F32, BF16, F16])
@pytest.mark.parametrize("rows,wide,outputs", [(1, 1024, 23), (8, 1152, 31), (13, 1152, 20), (25, 1152, 18), (50, 1024, 19)])
def test_products_of_few_rows(driver, mode, rows, wide, outputs):  # noqa: F811
    driver("scales", mode, rows, wide, outputs, 0, -1)


@pytest.mark.parametrize("mode,tile", [(BF16, 1), (F16, 2), (F32, 2), (F32, 3), (F32, 4), (F32, 5)])
@pytest.mark.parametrize("rows,wide,outputs", [(9, 1152, 20), (70, 256, 130)])
def test_products_by_tiles(driver, mode, tile, rows, wide, outputs):  # noqa: F811
    driver("scales", mode, rows, wide, outputs, 0, tile)


def test_products_of_few_rows_and_many_outputs_with_fp32_results(driver):  # noqa: F811
    """Several groups of rows of the weights a workgroup, which only fp32 results take with so many rows."""
    driver("scales", F32, 18, 1024, 8193, 0, -1)
