"""Top logits of rows whose list lies far above all others, as a sure teacher's or a low temperature's do: the logarithm of the others'
sum at every distance, against its definition in 64 bits.  Needs a GPU."""
import math

import pytest
import torch

import teacher_reference as R
from test_gpu_teacher import L, MODES, blocks, check_distill, check_top, noise  # noqa: F401

pytestmark = pytest.mark.gpu
# in temperatures: next to where sums of 2^-32 end (15 to 23), and those of fp32 (88 and more)
APART = [10, 14, 15, 16, 18, 20, 22, 24, 26, 28, 40, 90]


def rows_apart(columns, k, temperature):
    """Of each distance three rows: k logits about zero and the others that far below, all equal, one of them 5 temperatures above the rest,
    and as noise."""
    random = noise(columns + k, 3 * len(APART), columns)
    z = torch.empty_like(random)
    for i, apart in enumerate(APART):
        z[3 * i] = -apart
        z[3 * i + 1] = -apart - 5
        z[3 * i + 1, columns // 2] = -apart
        z[3 * i + 2] = random[3 * i + 2] - apart
    for r in range(len(z)):
        listed = torch.randperm(columns, generator=torch.Generator().manual_seed(r))[:k]
        listed = listed[listed != columns // 2]
        z[r, listed] = random[r, listed].abs() / 4
    return z * temperature


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("temperature", [0.2, 2.0])
@pytest.mark.parametrize("columns,k", [(100, 1), (300, 64), (1000, 1), (1000, 64), (2000, 33), (5000, 1), (5000, 100), (16001, 64), (50021, 1), (50021, 64), (66001, 20),
                                       (140001, 64)])
def test_others_far_below_the_list(blocks, mode, columns, k, temperature):  # noqa: F811
    check_top(blocks[mode], rows_apart(columns, k, temperature).to(R.DTYPES[mode]).cuda(), k, temperature)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("columns", [1000, 20000])
def test_others_of_noise_at_a_low_temperature(blocks, mode, columns):  # noqa: F811
    for temperature in (0.05, 0.1, 0.2, 0.4):
        check_top(blocks[mode], noise(columns, 8, columns).to(R.DTYPES[mode]).cuda(), 1, temperature)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("columns", [1000, 66001])
def test_infinities_and_nans_beside_others_far_below(blocks, mode, columns):  # noqa: F811
    """The list has the infinities, or all but one; a NaN makes the logarithm none."""
    z = torch.full((4, columns), -22.0, dtype=torch.float64)
    z[:, 3] = 0.0
    z[1, 7] = math.inf
    z[2, [7, 8]] = math.inf
    z[3, 11] = math.nan
    for k in (1, 2):
        check_top(blocks[mode], z.to(R.DTYPES[mode]).cuda(), k)


@pytest.mark.parametrize("mode", MODES)
def test_a_row_far_above_its_others_is_the_same_in_any_batch(blocks, mode):  # noqa: F811
    k, d, columns = 64, R.DTYPES[mode], 3001
    z = rows_apart(columns, k, 1.0).to(d).cuda().repeat(9, 1)
    whole = None
    for rows in (list(range(len(z))), [3], list(range(20))):
        new = lambda t, *shape: torch.zeros(shape, dtype=t, device="cuda")  # noqa: E731
        made = new(torch.int32, len(rows), k), new(torch.float32, len(rows), k), new(torch.float32, len(rows))
        blocks[mode].top(z[rows].contiguous(), *made[:2], rest=made[2], temperature=1.0)
        whole = whole or made
        for t, of in zip(made, whole):
            assert torch.equal(t.view(torch.int32), of[rows].contiguous().view(torch.int32))


@pytest.mark.parametrize("mode", MODES)
def test_a_student_of_a_sure_teacher(blocks, mode):  # noqa: F811
    """The distance from what top gives of such rows: p of the rest is next to nothing, and counts."""
    k, d, columns, rows = 3, R.DTYPES[mode], 900, 3 * len(APART)
    teacher = rows_apart(columns, k, 1.0).to(d).cuda()
    index, value = torch.zeros(rows, k, dtype=torch.int32, device="cuda"), torch.zeros(rows, k, device="cuda")
    rest = torch.zeros(rows, device="cuda")
    blocks[mode].top(teacher, index, value, rest=rest)
    want = R.top(teacher, k, 1.0)
    z = noise(5, rows, columns, std=2.0).to(d).cuda()
    distance = R.distill(z, *want, 1.0, None, 1.0)
    check_distill(blocks[mode], mode, z, index.cpu(), value.cpu(), rest.cpu(), 1.0, want=distance)
