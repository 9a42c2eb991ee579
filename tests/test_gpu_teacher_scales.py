"""Products of packed matrices whose blocks have scales next to the ends of what is allowed, 2^-127 and 2^127, against their
definition in 64 bits.  Needs a GPU."""
import math

import pytest
import torch

import teacher_reference as R
from test_gpu_teacher import L, MODES, blocks, guarded, noise, packed, untouched  # noqa: F401

pytestmark = pytest.mark.gpu
CENTRES = [0, 3, 8, 11, 60, 127, 200, 245, 248, 254]      # next to where numbers of 8 bits leave bfloat16's range, 10 and 246


def matrix(seed, rows, wide, centres):
    """Numbers of 8 bits of every size, and a row's scales next to its centre."""
    g = torch.Generator().manual_seed(seed)
    bits = torch.randint(0, 127, (rows, wide), generator=g) + 128 * torch.randint(0, 2, (rows, wide), generator=g)
    count = wide // 128
    scale = torch.full((rows, -(-count // 4) * 4), 127)
    scale[:, :count] = (torch.tensor(centres)[torch.arange(rows) % len(centres)][:, None] + torch.randint(-2, 3, (rows, count), generator=g)).clamp(0, 254)
    return bits.to(torch.uint8).cuda(), scale.to(torch.uint8).cuda()


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("rows,wide,outputs", [(1, 128, 10), (2, 128, 11), (9, 640, 23), (1, 1152, 20), (4, 1152, 31), (8, 1024, 40), (13, 1152, 24), (24, 1152, 70), (60, 1152, 33), (3, 1152, 8195), (12, 1152, 8197), (20, 1152, 8195),
                                               (70, 128, 30), (80, 640, 70), (300, 384, 140)])
def test_product_with_scales_next_to_their_ends(blocks, mode, rows, wide, outputs):  # noqa: F811
    """Every pair of ends; compared are those whose products a number of the results' type can hold."""
    x, xs = matrix(rows + wide, rows, wide, CENTRES)
    w, ws = matrix(outputs, outputs, wide, CENTRES[::-1])
    y, room = guarded(rows, outputs, R.DTYPES[mode], 1)
    blocks[mode].packed_product(x, xs, w, ws, y)
    torch.cuda.synchronize()
    assert untouched(room, y)
    vx, vw = R.values(x, xs), R.values(w, ws)
    want, off = R.product(vx, vw, mode)
    # next to zero each addition's rounding is up to half of fp32's least step
    off = off + wide * 2.0 ** -150
    size = vx.abs() @ vw.abs().t()
    most = 60000.0 if mode == "f16" else 2.0 ** 127
    fits, got = size < most, y.double().cpu()
    assert int(fits.sum()) >= fits.numel() // 4
    assert bool(((got - want).abs() <= off)[fits].all()), float((((got - want).abs() / off)[fits]).max())


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("rows,wide", [(3, 128), (5, 1152), (20, 1152), (90, 128)])
def test_numbers_that_cancel_with_the_scales(blocks, mode, rows, wide):  # noqa: F811
    """4 2^127 by 2^-127 is 4, 2^-9 2^-127 by 2^127 is 2^-9: neither is a bfloat16 number on its own side.  Two that are too large are
    an infinity of their sign, and a NaN or a block that is none stays one."""
    count = wide // 128
    x, w = torch.zeros(rows, wide, dtype=torch.uint8, device="cuda"), torch.zeros(6, wide, dtype=torch.uint8, device="cuda")
    xs, ws = (torch.full((n, -(-count // 4) * 4), 127, dtype=torch.uint8, device="cuda") for n in (rows, 6))
    x[:, 0], xs[:, :count] = 0x48, 254                   # 4
    x[1, 0], xs[1, :count] = 0x01, 0                     # 2^-9
    w[:, 0] = 0x38                                       # 1
    ws[0, :count] = 0
    ws[1, :count] = 254
    w[2, 0], ws[2, :count] = 0xB8, 254                   # -1
    ws[3, 0] = 255
    w[4, 5], ws[4, :count] = 0x7F, 0
    y = torch.zeros(rows, 6, dtype=R.DTYPES[mode], device="cuda")
    blocks[mode].packed_product(x, xs, w, ws, y)
    y = y.double().cpu()
    large = torch.arange(rows) != 1
    assert bool((y[large, 0] == 4.0).all())
    assert float(y[1, 1]) == 2.0 ** -9 and float(y[1, 2]) == -2.0 ** -9
    assert bool((y[large, 1] == math.inf).all()) and bool((y[large, 2] == -math.inf).all())
    assert bool(torch.isnan(y[:, 3:5]).all())
    # (2^129: past fp32 and bfloat16 too)
    assert bool((y[large, 5] == math.inf).all())


def test_a_product_is_the_same_beside_scales_at_their_ends(blocks):  # noqa: F811
    """Rows of ordinary scales have the bits that they have without neighbours of others."""
    wide, outputs, rows = 640, 200, 300
    x, xs = matrix(1, rows, wide, [120, 127, 131])
    w, ws = matrix(2, outputs, wide, [120, 127, 131])
    for mode in MODES:
        alone, beside = (torch.zeros(rows, outputs, dtype=R.DTYPES[mode], device="cuda") for _ in range(2))
        blocks[mode].packed_product(x, xs, w, ws, alone)
        far_x, far_w = xs.clone(), ws.clone()
        far_x[7::20], far_w[3::17] = 254, 1
        blocks[mode].packed_product(x, far_x, w, far_w, beside)
        same_x, same_w = torch.arange(rows) % 20 != 7, torch.arange(outputs) % 17 != 3
        assert torch.equal(alone.cpu()[same_x][:, same_w], beside.cpu()[same_x][:, same_w])


def test_largest_and_smallest_numbers_through_packed_matrices(L, blocks):  # noqa: F811
    """What quantise makes of fp32's ends, by what brings it back."""
    for size, back in ((3.3e38, 2.0 ** -100), (2.0 ** -135, 2.0 ** 100)):
        for rows in (3, 70):
            x = (noise(1, rows, 300).clamp(-1, 1) * size).float().cuda()
            w = (noise(2, 20, 300).clamp(-1, 1) * back).float().cuda()
            q, qs = packed(L, blocks, "f32", x)
            p, ps = packed(L, blocks, "f32", w)
            y = torch.zeros(rows, 20, device="cuda")
            blocks["f32"].packed_product(q, qs, p, ps, y)
            want, off = R.product(R.values(q, qs), R.values(p, ps), "f32")
            assert bool(((y.double().cpu() - want).abs() <= off).all())
