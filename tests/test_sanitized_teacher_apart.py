"""As test_sanitized_teacher_kernels.py: rows whose listed logits lie far above all others, as a sure teacher's do, so that the others'
sum is next to nothing beside the list's."""
import pytest

from test_sanitized_teacher_kernels import BF16, F16, F32, driver  # noqa: F401


# (distances, in temperatures, next to where sums of 2^-32 and of fp32 end; below zero: one of the others lies 5 above the rest of them)
@pytest.mark.parametrize("kind", [10, 14, 15, 18, 20, 22, 24, 26, 28, 40, 90, -10, -15, -18, -20, -22, -24, -28, -40, -90])
@pytest.mark.parametrize("mode,columns,k", [(F32, 300, 1), (F16, 1000, 20), (BF16, 3001, 1), (F32, 2500, 64)])
def test_top_of_rows_whose_list_lies_far_above(driver, mode, columns, k, kind):  # noqa: F811
    driver("top", mode, 1, columns, k, 0, kind)


@pytest.mark.parametrize("kind", [15, 22, -20])
@pytest.mark.parametrize("mode,columns,k", [(BF16, 16000, 100), (F32, 66001, 20), (F16, 132000, 7)])
def test_top_of_long_rows_whose_list_lies_far_above(driver, mode, columns, k, kind):  # noqa: F811
    driver("top", mode, 1, columns, k, 0, kind)
