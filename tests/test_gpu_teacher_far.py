"""Distillation from a teacher whose logits lie far from zero, or whose temperature takes them past fp32's range: what counts are their
distances.  Needs a GPU."""
import math

import pytest
import torch

import teacher_reference as R
from test_gpu_teacher import L, MODES, blocks, check_distill, lists, noise  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("columns,k", [(200, 1), (900, 20), (900, 100), (70001, 20)])
@pytest.mark.parametrize("offset,temperature", [(10000.0, 0.7), (-10000.0, 0.7), (3e4, 3.0), (2.0 ** 100, 1.5), (-3.0e38, 0.7), (3.0e38, 0.7), (1.0, 1e-38), (-1.0, 1e-38)])
def test_lists_far_from_zero(blocks, mode, columns, k, offset, temperature):  # noqa: F811
    """The list alone: p is the softmax of the values' distances.  Even with a temperature next to zero p and, where the student is sure
    of nothing, the gradient are numbers."""
    rows = 4
    index, value = lists(k, rows, columns, k)
    value = (value.double() + offset).float()
    z = noise(columns, rows, columns) if temperature > 1e-30 else torch.zeros(rows, columns, dtype=torch.float64)
    check_distill(blocks[mode], mode, z.to(R.DTYPES[mode]).cuda(), index, value, None, temperature, None, min(1.0, temperature))


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("temperature", [0.5, 1e-38])
def test_a_rest_beside_values_past_the_range(blocks, mode, temperature):  # noqa: F811
    """Values that the temperature takes past fp32's range are all or nothing beside a rest within it; one that is -infinity is none, an
    infinity makes no number."""
    columns, k, d = 300, 3, R.DTYPES[mode]
    index, _ = lists(1, 5, columns, k)
    value = torch.full((5, k), 3.0e38)
    value[1], value[3] = -3.0e38, -3.0e38
    rest = torch.tensor([2.0, 2.0, -math.inf, -math.inf, math.inf])
    z = torch.zeros(5, columns, dtype=d, device="cuda")
    loss, dz = torch.zeros(5, device="cuda"), torch.zeros(5, columns, dtype=d, device="cuda")
    blocks[mode].distill(z, index.cuda(), value.cuda(), loss, dz, rest=rest.cuda(), temperature=temperature, scale=temperature)
    loss, dz = loss.double().cpu() / temperature, dz.double().cpu()
    # p is 1 / k for each of the list, or one for all others; the student's are 1 / columns each
    off = 400 * R.U
    for r, want in ((0, math.log(columns / k)), (1, -math.log((columns - k) / columns)), (2, math.log(columns / k)), (3, math.log(columns / k))):
        assert abs(float(loss[r]) - want) <= off * (1 + want), r
        listed = torch.zeros(columns, dtype=torch.bool)
        listed[index[r].long()] = True
        p = torch.where(listed, 1.0 / k, 0.0) if r != 1 else torch.where(listed, 0.0, 1.0 / (columns - k))
        want_dz = (1.0 / columns - p.double())
        assert bool(((dz[r] - want_dz).abs() <= (off + R.HALF_STEP[mode]) * (1.0 / columns + p)).all()), r
    assert bool(torch.isnan(loss[4])) and bool(torch.isnan(dz[4]).all())


@pytest.mark.parametrize("mode", MODES)
def test_a_row_masked_by_the_lowest_number_at_a_low_temperature(blocks, mode):  # noqa: F811
    """A teacher that has nothing left says so of as many columns as it lists, all alike."""
    columns, k, d = 500, 8, R.DTYPES[mode]
    teacher = torch.full((2, columns), torch.finfo(d).min, dtype=d, device="cuda")
    index, value = torch.zeros(2, k, dtype=torch.int32, device="cuda"), torch.zeros(2, k, device="cuda")
    blocks[mode].top(teacher, index, value, temperature=0.5)
    z = noise(3, 2, columns).to(d).cuda()
    got, _ = check_distill(blocks[mode], mode, z, index.cpu(), value.cpu(), None, 0.5)
    assert bool((got > 0).all())
