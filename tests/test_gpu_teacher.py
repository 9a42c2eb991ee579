"""Packed matrices, their product, top logits and distillation against their definitions in 64 bits, at the sizes, masks and
values where they can go wrong.  Needs a GPU."""
import math

import pytest
import torch

import teacher_reference as R

pytestmark = pytest.mark.gpu
MODES = ["f32", "bf16", "f16"]


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    torch.cuda.set_device(0)
    import paper_1805_01993_amd as lib
    lib.load_library()
    return lib


@pytest.fixture(scope="module")
def blocks(L):
    return {mode: L.ccdc_block(8, 1, mode).bind([3]).upload() for mode in MODES}


def guarded(rows, columns, dtype, pad=0, ahead=0, fill=7):
    """A [rows][columns] view with `pad` elements between rows and `ahead` before the first, and all there is around it."""
    room = torch.full((ahead + rows * (columns + pad) + 64,), fill, device="cuda").to(dtype)
    return room[ahead:ahead + rows * (columns + pad)].view(rows, columns + pad)[:, :columns], room


def untouched(room, view, fill=7):
    """Whether the bytes around a view still are what they were."""
    mask = torch.ones(room.shape, dtype=torch.bool, device="cuda")
    mask.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(False)
    want = torch.full((1,), fill, device="cuda").to(room.dtype)
    return bool((room[mask].view(torch.uint8 if room.element_size() == 1 else room.dtype) == want.view(torch.uint8 if room.element_size() == 1 else room.dtype)).all())


def noise(seed, *shape, std=1.0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * std


# ------------------------------------------------------------------ packed matrices
def packed(L, blocks, mode, x, ahead=0):
    """A matrix packed by the library, with room around what it writes."""
    rows, columns = x.shape
    (_, wide), (_, kept) = L.packed_shapes(rows, columns)
    q, room_q = guarded(rows, wide, torch.uint8, fill=9)
    scale, room_s = guarded(rows, kept, torch.uint8, fill=9)
    blocks[mode].quantise(x, q.view(torch.float8_e4m3fn), scale)
    torch.cuda.synchronize()
    assert untouched(room_q, q, 9) and untouched(room_s, scale, 9)
    return q, scale


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("rows,columns,pad,ahead", [(1, 1, 0, 0), (3, 127, 0, 0), (5, 128, 8, 0), (7, 129, 3, 1), (4, 2001, 0, 5), (33, 515, 1, 0), (2, 9000, 0, 0)])
def test_quantise(L, blocks, mode, rows, columns, pad, ahead):
    x, _ = guarded(rows, columns, R.DTYPES[mode], pad, ahead)
    values = noise(1, rows, columns) * torch.exp2(torch.randint(-12, 9, (rows, columns), generator=torch.Generator().manual_seed(2)).double())
    x.copy_(values)
    q, scale = packed(L, blocks, mode, x)
    want_q, want_scale = R.quantise(x.double())
    assert torch.equal(scale.cpu(), want_scale)
    assert torch.equal(q.cpu(), want_q)


@pytest.mark.parametrize("mode", MODES)
def test_quantise_values_at_their_limits(L, blocks, mode):
    """Zeros, the smallest and largest numbers, a block's largest at 448 of a power and next to it, ties, infinities and NaNs."""
    info, d = torch.finfo(R.DTYPES[mode]), R.DTYPES[mode]
    x = torch.zeros(12, 256, dtype=torch.float64)
    x[1, :3] = torch.tensor([-0.0, 0.0, info.tiny])
    x[2, 5] = info.smallest_normal * info.eps                       # the smallest number
    x[3, :4] = torch.tensor([info.max, -info.max, 1.0, info.tiny])
    x[4, :3] = torch.tensor([448.0, 1.0, -448.0])
    x[5, :3] = torch.tensor([448.0 * (1 + info.eps), 1.0, 3.0])
    x[6, :3] = torch.tensor([7.0 / 16, 1.0 / 16, -0.4])
    x[7] = torch.linspace(1, 448, 256, dtype=torch.float64)
    x[8, :128] = torch.arange(128) * 0.0625 + 1.0625                # half way between two numbers of 8 bits
    x[8, 127] = 448.0
    x[9, :4] = torch.tensor([math.inf, 3.0, -math.inf, math.nan])
    x[9, 200] = math.nan
    x[10, :128] = math.inf
    x[11, 0] = 1.0
    x[11, 1:60] = 2.0 ** -9 * torch.arange(59) / 16                # below the smallest of 8 bits at this scale
    x = x.to(d).cuda()
    q, scale = packed(L, blocks, mode, x)
    want_q, want_scale = R.quantise(x.double())
    assert torch.equal(scale.cpu(), want_scale)
    nan = torch.isnan(x.cpu())
    got, want = q.cpu(), want_q
    assert torch.equal(got[~nan], want[~nan]) and bool(((got[nan] & 127) == 127).all())


# ------------------------------------------------------------------ their product
def random_packed(seed, rows, wide, spread=6):
    """Numbers of 8 bits as blocks of a matrix have them, and scales that differ."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, wide, generator=g, dtype=torch.float64) * torch.exp2(torch.randint(-spread, 1, (rows, wide // 128, 1), generator=g).double()).expand(-1, -1, 128).reshape(rows, wide)
    bits, scale = R.quantise(x)
    return bits.cuda(), scale.cuda()


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("rows,wide,outputs,pad", [
    (1, 128, 1, 0), (1, 256, 5, 0), (2, 640, 33, 3), (4, 1152, 64, 0), (5, 128, 16, 0), (8, 896, 17, 1), (9, 384, 70, 0), (16, 1280, 15, 0),
    (17, 256, 40, 0), (32, 512, 31, 2), (33, 128, 100, 0), (64, 768, 65, 0),                      # to the matrix instructions from memory
    (65, 128, 1, 0), (65, 256, 130, 0), (129, 384, 127, 5), (130, 512, 129, 0), (300, 640, 77, 0), (70, 1152, 260, 3)])   # by tiles
def test_product(blocks, mode, rows, wide, outputs, pad):
    x, xs = random_packed(rows + wide, rows, wide)
    w, ws = random_packed(outputs + wide, outputs, wide)
    y, room = guarded(rows, outputs, R.DTYPES[mode], pad)
    blocks[mode].packed_product(x, xs, w.view(torch.float8_e4m3fn), ws, y)
    torch.cuda.synchronize()
    want, off = R.product(R.values(x, xs), R.values(w, ws), mode)
    assert bool(((y.double().cpu() - want).abs() <= off).all()), float(((y.double().cpu() - want).abs() / off).max())
    assert untouched(room, y)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("rows", [1, 4, 5, 8, 9, 16, 17, 32, 33, 64])
@pytest.mark.parametrize("wide,outputs", [(1024, 50), (1152, 2047), (1664, 2050), (2176, 8195)])
def test_product_of_few_rows(blocks, mode, rows, wide, outputs):
    """The kernels that take the weights from memory to the matrix instructions, with parts of k that end before others, groups of rows
    past the last, and more workgroups of two groups; all columns of some rows of the weights where these are many."""
    x, xs = random_packed(rows + wide, rows, wide)
    w, ws = random_packed(outputs, outputs, wide)
    ws[:, wide // 128:] = 255                     # bytes past the last block say nothing
    y, room = guarded(rows, outputs, R.DTYPES[mode], 1)
    blocks[mode].packed_product(x, xs, w, ws, y)
    torch.cuda.synchronize()
    assert untouched(room, y)
    picked = torch.unique(torch.cat((torch.arange(0, outputs, 1 + outputs // 60), torch.arange(max(0, outputs - 20), outputs))))
    want, off = R.product(R.values(x, xs), R.values(w[picked.cuda()], ws[picked.cuda()]), mode)
    got = y.double().cpu()[:, picked]
    assert bool(((got - want).abs() <= off).all()), float(((got - want).abs() / off).max())


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("rows", [9, 16, 17, 31, 33, 47, 64])
@pytest.mark.parametrize("outputs", [7, 500, 1021, 1500, 2048, 4093, 4100])
def test_product_of_few_rows_divided_among_workgroups(blocks, mode, rows, outputs):
    """Groups of 8, 16 and 32 rows, the last of them not full; what is next to the result stays."""
    x, xs = random_packed(rows, rows, 1152)
    w, ws = random_packed(outputs, outputs, 1152)
    y, room = guarded(rows, outputs, R.DTYPES[mode], 1)
    blocks[mode].packed_product(x, xs, w, ws, y)
    torch.cuda.synchronize()
    assert untouched(room, y)
    want, off = R.product(R.values(x, xs), R.values(w, ws), mode)
    assert bool(((y.double().cpu() - want).abs() <= off).all()), float(((y.double().cpu() - want).abs() / off).max())


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("rows,wide,outputs", [(2049, 128, 4100), (4096, 256, 2304), (1030, 384, 5003), (700, 2304, 900)])
def test_products_of_many_tiles(blocks, mode, rows, wide, outputs):
    """Tiles of both sizes, with edges; compared where the definition is affordable: some rows, some columns."""
    x, xs = random_packed(1, rows, wide)
    w, ws = random_packed(2, outputs, wide)
    y, room = guarded(rows, outputs, R.DTYPES[mode], 1)
    blocks[mode].packed_product(x, xs, w, ws, y)
    torch.cuda.synchronize()
    assert untouched(room, y)
    y, vx, vw = y.double().cpu(), R.values(x, xs), R.values(w, ws)
    for picked_x, picked_w in ((torch.arange(rows), torch.arange(0, outputs, 97)), (torch.arange(0, rows, 89), torch.arange(outputs))):
        want, off = R.product(vx[picked_x], vw[picked_w], mode)
        got = y[picked_x][:, picked_w]
        assert bool(((got - want).abs() <= off).all()), float(((got - want).abs() / off).max())


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("rows,wide", [(1, 512), (20, 512), (100, 512), (1, 1152), (7, 1152), (16, 1664), (30, 1152), (60, 1664)])
def test_product_of_what_is_no_number(blocks, mode, rows, wide):
    """A NaN, and a block that is none, reach their own row or column and no other; zeros against them are none either."""
    x, xs = random_packed(1, rows, wide)
    w, ws = random_packed(2, 40, wide)
    x[rows - 1, 300] = 0x7F
    w[3, 17] = 0xFF
    ws[7, 2] = 255
    ws[:, wide // 128:] = 255                     # bytes past the last block say nothing
    y = torch.zeros(rows, 40, dtype=R.DTYPES[mode], device="cuda")
    blocks[mode].packed_product(x, xs, w, ws, y)
    want = torch.zeros(rows, 40, dtype=torch.bool)
    want[rows - 1] = want[:, 3] = want[:, 7] = True
    assert torch.equal(torch.isnan(y).cpu(), want)


def test_product_at_the_scales_limits(blocks):
    """Scales of 2^-127 and 2^127 that cancel, and what is too large for the results."""
    for rows in (2, 80):
        x = torch.full((rows, 128), 0x38, dtype=torch.uint8, device="cuda")
        w = x[:2].clone()
        xs, ws = (torch.full((n, 4), 127, dtype=torch.uint8, device="cuda") for n in (rows, 2))
        xs[:, 0], ws[:, 0] = 254, 0
        y = torch.zeros(rows, 2, dtype=torch.bfloat16, device="cuda")
        blocks["bf16"].packed_product(x, xs, w, ws, y)
        assert bool((y == 128).all())
        ws[1, 0] = 254
        blocks["bf16"].packed_product(x, xs, w, ws, y)
        assert bool((y[:, 0] == 128).all()) and bool(torch.isinf(y[:, 1]).all())


# ------------------------------------------------------------------ top logits
def check_top(block, z, k, temperature=1.0, with_rest=True):
    rows, columns = z.shape
    index, room_i = guarded(rows, k, torch.int32)
    value, room_v = guarded(rows, k, torch.float32)
    rest, room_r = guarded(1, rows, torch.float32)
    block.top(z, index, value, rest=rest[0] if with_rest else None, temperature=temperature)
    torch.cuda.synchronize()
    assert untouched(room_i, index) and untouched(room_v, value) and untouched(room_r, rest)
    want_index, want_value, want_rest = R.top(z, k, temperature)
    assert torch.equal(index.cpu(), want_index)
    assert torch.equal(value.double().cpu(), want_value)
    if not with_rest:
        return bool((rest == 7).all())
    got = rest[0].double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want_rest)) and torch.equal(torch.isinf(got), torch.isinf(want_rest))
    fine = torch.isfinite(want_rest)
    # roundings of the sum (a thread's share, the wavefronts'), of exponentials' arguments where they count, and of what is summed from
    off = (400 + columns / 1024) * R.U * (1 + want_rest.abs() + z.double().cpu().nan_to_num(0, 0, 0).abs().amax(1) / temperature)
    assert bool(((got - want_rest).abs() <= off)[fine].all())


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("rows,columns,k,temperature,pad", [
    (1, 1, 1, 1.0, 0), (3, 5, 8, 0.5, 0), (2, 8, 8, 1.0, 1), (5, 100, 1, 2.0, 0), (4, 512, 128, 1.0, 0), (3, 513, 9, 1.0, 7), (6, 1000, 100, 1.0, 0),
    (2, 1025, 64, 0.7, 0), (3, 4096, 128, 1.0, 8), (2, 4097, 3, 1.0, 0), (2, 8200, 50, 1.5, 0), (2, 16385, 128, 1.0, 1), (2, 32768, 64, 1.0, 0),
    (1, 50021, 40, 2.0, 0), (2, 65537, 128, 1.0, 0), (1, 140001, 20, 1.0, 0)])
def test_top(blocks, mode, rows, columns, k, temperature, pad):
    z, _ = guarded(rows, columns, R.DTYPES[mode], pad)
    z.copy_(noise(columns + k, rows, columns, std=3.0))
    check_top(blocks[mode], z, k, temperature)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("columns", [90, 1000, 5000, 20000, 70001])
def test_top_of_equal_and_masked_logits(blocks, mode, columns):
    """Ties of all, ties at the border of the list, zeros of both signs, rows that are masked but for few columns or altogether, the
    lowest number as a mask, logits in order, NaNs and infinities."""
    d, k = R.DTYPES[mode], 64
    z = noise(columns, 14, columns).to(d).double()
    z[0] = 0.25
    z[1] = torch.where(torch.arange(columns) % 2 == 0, 0.0, -0.0)
    z[2] = torch.round(z[2])
    z[3] = -math.inf
    z[4, :] = -math.inf
    z[4, columns - 3:] = torch.tensor([1.0, -2.0, 1.0])
    z[5, 10:] = torch.finfo(d).min
    z[6] = torch.arange(columns).double() / columns
    z[7] = -torch.arange(columns).double() / columns
    z[8, 3] = math.nan
    z[9, columns // 2] = math.inf
    z[10] = torch.finfo(d).min
    z[11, :] = -1000.0                                 # so far below the list that fp32's exponentials are zero
    z[11, :k] = 1000.0
    z[12, columns // 3:] = 5.0                         # more of the same than the list in LDS has room for
    z[13] = math.nan
    z = z.to(d).cuda()
    check_top(blocks[mode], z, k)
    check_top(blocks[mode], z, 1, 0.5, with_rest=False)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("columns", [500, 999, 1801, 3501, 8000, 16001, 32001, 50021, 70001])
def test_a_row_is_the_same_every_time_and_in_any_batch(blocks, mode, columns):
    """Nodes that store a file make the same bits of its rows, whatever else is in their batches, how many rows they have and what
    addresses the rows begin at."""
    block, k, d = blocks[mode], 20, R.DTYPES[mode]
    z = noise(4, 300, columns, std=2.0).to(d).cuda()
    whole = None
    for rows in (list(range(300)), list(range(300)), [7], [299, 7, 120]):
        part = z[rows].contiguous()
        new = lambda t, *shape: torch.zeros(shape, dtype=t, device="cuda")  # noqa: E731
        made = {"index": new(torch.int32, len(rows), k), "value": new(torch.float32, len(rows), k), "rest": new(torch.float32, len(rows)),
                "loss": new(torch.float32, len(rows)), "dz": new(d, len(rows), columns)}
        block.top(part, made["index"], made["value"], rest=made["rest"], temperature=1.5)
        # (the neighbour's answer, so that something is left to learn)
        index, value = made["index"].roll(3, 1).contiguous(), made["value"].contiguous()
        block.distill(part, index, value, made["loss"], made["dz"], rest=made["rest"], temperature=1.5)
        whole = whole or made
        for name, t in made.items():
            assert torch.equal(t.view(torch.uint8), whole[name][rows].contiguous().view(torch.uint8)), (name, len(rows))


# ------------------------------------------------------------------ distillation
def check_distill(block, mode, z, index, value, rest=None, temperature=1.0, weight=None, scale=1.0, pad=0, place=False, want=None):
    rows, columns = z.shape
    d = R.DTYPES[mode]
    want_loss, want_dz, off_loss, off_dz = want or R.distill(z, index, value, rest, temperature, weight, scale)
    on = lambda t, dtype: None if t is None else t.to(dtype).cuda().contiguous()  # noqa: E731
    index, value, rest, weight = on(index, torch.int32), on(value, torch.float32), on(rest, torch.float32), on(weight, torch.float32)
    loss, room_l = guarded(1, rows, torch.float32)
    dz, room_z = guarded(rows, columns, d, pad)
    if place:
        dz.copy_(z)
        z = dz
    block.distill(z, index, value, loss[0], dz, rest=rest, temperature=temperature, weight=weight, scale=scale)
    torch.cuda.synchronize()
    assert untouched(room_l, loss) and untouched(room_z, dz)
    got, got_dz = loss[0].double().cpu(), dz.double().cpu()
    for a, b, off, dtype in ((got, want_loss, off_loss, torch.float32), (got_dz, want_dz, off_dz + R.HALF_STEP[mode] * want_dz.abs() + R.SMALLEST[mode], d)):
        # what is larger than the type's largest number is an infinity in it (a listed column at -3.4e38 costs 2 x 3.4e38 / 1.3 p)
        b = torch.where(b.abs() > torch.finfo(dtype).max, b.sign() * math.inf, b)
        assert torch.equal(torch.isnan(a), torch.isnan(b))
        assert torch.equal(a[torch.isinf(b)], b[torch.isinf(b)])
        fine = torch.isfinite(b)
        assert bool(((a - b).abs() <= off + R.U * b.abs())[fine].all()), float(((a - b).abs() / (off + 1e-300))[fine].max())
    alone = torch.full((rows,), 5.0, device="cuda")
    if not place:
        block.distill(z, index, value, alone, None, rest=rest, temperature=temperature, weight=weight, scale=scale)
        assert torch.equal(alone.view(torch.int32), loss[0].contiguous().view(torch.int32))
        again = torch.empty_like(dz)
        block.distill(z, index, value, None, again, rest=rest, temperature=temperature, weight=weight, scale=scale)
        assert torch.equal(again.view(torch.uint8), dz.contiguous().view(torch.uint8))
    return got, got_dz


def lists(seed, rows, columns, k):
    """Distinct columns of each row and the teacher's logits there."""
    g = torch.Generator().manual_seed(seed)
    index = torch.stack([torch.randperm(columns, generator=g)[:k] for _ in range(rows)])
    if index.shape[1] < k:
        index = torch.nn.functional.pad(index, (0, k - index.shape[1]), value=-1)
    return index.int(), torch.randn(rows, k, generator=g) * 2


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("rows,columns,k,temperature,rest,pad", [
    (1, 1, 1, 1.0, False, 0), (2, 3, 5, 1.0, True, 0), (3, 8, 2, 0.5, True, 1), (4, 100, 128, 1.0, True, 0), (2, 511, 1, 1.0, False, 0),
    (2, 512, 64, 2.0, True, 8), (3, 1000, 65, 1.0, False, 0), (2, 1025, 128, 3.0, True, 3), (2, 4096, 20, 1.0, True, 0), (1, 4104, 20, 0.7, False, 0),
    (2, 8193, 7, 1.0, True, 1), (1, 16384, 128, 1.0, True, 0), (2, 32770, 33, 2.0, True, 0), (1, 65536, 64, 1.0, False, 0),
    (2, 70001, 64, 1.0, True, 0), (1, 131072, 10, 1.5, True, 0)])
def test_distill(blocks, mode, rows, columns, k, temperature, rest, pad):
    z = noise(columns, rows, columns, std=2.0).to(R.DTYPES[mode]).cuda()
    index, value = lists(k, rows, columns, k)
    all_listed = bool((k >= columns))
    rest = noise(3, rows).float() if rest and not all_listed else None
    weight = torch.rand(rows, generator=torch.Generator().manual_seed(1)) + 0.5
    want = R.distill(z, index, value, rest, temperature, weight, 64.0)
    for place in (False, True):
        check_distill(blocks[mode], mode, z, index, value, rest, temperature, weight, 64.0, pad, place, want)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("columns", [70, 3000, 40000, 66000])
def test_distill_rows_of_every_kind(blocks, mode, columns):
    """Masked logits, whole rows masked, empty and short lists, indexes out of range and twice, weights of zero over rows that are no
    numbers, listed columns that have everything or nothing."""
    d, rows, k = R.DTYPES[mode], 18, 12
    z = noise(columns, rows, columns).to(d).double()
    index, value = lists(5, rows, columns, k)
    rest, weight = noise(6, rows).float(), torch.ones(rows)
    z[0, 20:] = -math.inf                              # a padded end, and some of the list in it
    index[0] = torch.arange(k).int()
    z[1] = -math.inf                                   # nothing to choose from
    index[2] = -1                                      # no list
    value[3, 4:], index[3, 4:] = -math.inf, -1         # a short one
    index[4, 3], index[4, 4] = columns, -2147483648
    index[5, 7], index[5, 9] = index[5, 2], index[5, 2]
    index[6] = index[6, 0]
    weight[7], z[7, 3] = 0.0, math.nan
    weight[8], z[8] = 0.0, -math.inf
    z[9, index[9].long()] = 300.0                      # nearly all of the row is listed
    z[10, index[10].long()] = -300.0                   # nearly none
    rest[11] = -math.inf                               # the teacher's list is all
    value[12] = -math.inf                              # it says that the rest is all
    z[13] = torch.finfo(d).min
    z[14, 5:] = torch.finfo(d).min
    index[14] = torch.arange(k).int()
    z[15] += 10000.0                                   # far from zero
    rest[16] = 500.0
    value[17, 3] = 600.0
    z = z.to(d).cuda()
    got, _ = check_distill(blocks[mode], mode, z, index, value, rest, 1.3, weight, 2.0)
    for r in (1, 2, 7, 8):
        assert float(got[r]) == 0.0
    check_distill(blocks[mode], mode, z, index, value, None, 1.0, weight, 1.0, pad=1)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("columns", [200, 9000, 70000])
def test_distill_of_what_is_no_number(blocks, mode, columns):
    """NaNs and infinities: the rows they are in, and no others; a listed column that is masked costs an infinity."""
    d, rows, k = R.DTYPES[mode], 7, 4
    z = noise(1, rows, columns).to(d).cuda()
    index, value = lists(2, rows, columns, k)
    index[:] = torch.arange(10, 10 + k).int()
    rest = torch.zeros(rows)
    z[0, 150] = math.nan
    z[1, 11] = math.nan
    z[2, 150] = math.inf
    z[3, 11] = math.inf
    z[4, 11] = -math.inf
    value[5, 0] = math.nan
    loss, dz = torch.zeros(rows, device="cuda"), torch.zeros(rows, columns, dtype=d, device="cuda")
    blocks[mode].distill(z, index.cuda(), value.cuda(), loss, dz, rest=rest.cuda())
    loss, dz = loss.cpu(), dz.cpu()
    for r in (0, 1, 2, 3, 5):
        assert math.isnan(loss[r]) and bool(torch.isnan(dz[r]).all()), r
    assert loss[4] == math.inf and bool(torch.isfinite(dz[4]).all()) and float(dz[4, 11]) < 0
    assert bool(torch.isfinite(loss[6])) and bool(torch.isfinite(dz[6]).all())


def test_gradient_against_differences(blocks):
    """Along directions, the change of the definition's loss is the gradient's product with them."""
    rows, columns, k = 3, 700, 20
    z = noise(1, rows, columns, std=2.0).float()
    index, value = lists(2, rows, columns, k)
    rest = noise(3, rows).float()
    dz, loss = torch.zeros(rows, columns, device="cuda"), torch.zeros(rows, device="cuda")
    blocks["f32"].distill(z.cuda(), index.cuda(), value.cuda(), loss, dz, rest=rest.cuda(), temperature=1.5, scale=2.0)
    of = lambda at: R.distill(at, index, value, rest, 1.5, None, 2.0)[0].sum()  # noqa: E731
    for seed in range(6):
        along, h = noise(seed, rows, columns), 1e-4
        change = (of(z.double() + h * along) - of(z.double() - h * along)) / (2 * h)
        # the third derivative's share is about h^2 |along|^3 / 6, the gradient's own error 400 roundings
        size = float((dz.double().cpu() * along).abs().sum())
        assert abs(float(change) - float((dz.double().cpu() * along).sum())) <= h * h * float(along.abs().max()) ** 3 * rows + 400 * R.U * (1 + size)


def test_cross_entropy_of_a_label(blocks):
    z = noise(1, 5, 333).float().cuda()
    label = torch.tensor([[0], [332], [5], [-1], [77]], dtype=torch.int32, device="cuda")
    value, loss, dz = torch.zeros(5, 1, device="cuda"), torch.zeros(5, device="cuda"), torch.zeros(5, 333, device="cuda")
    blocks["f32"].distill(z, label, value, loss, dz)
    zd = z.double().cpu().requires_grad_()
    want = torch.nn.functional.cross_entropy(zd, label[:, 0].long().cpu(), reduction="none", ignore_index=-1)
    (grad,) = torch.autograd.grad(want.sum(), zd)
    assert torch.allclose(loss.double().cpu(), want.detach(), rtol=400 * R.U, atol=400 * R.U)
    assert torch.allclose(dz.double().cpu(), grad, rtol=400 * R.U, atol=400 * R.U)


# ------------------------------------------------------------------ together, on streams, captured
def chain(block, x, W, W_scale, k, z, made, temperature=2.0):
    """A teacher's answer to x by its packed weights, and a student's distance from it."""
    block.quantise(x, made["q"], made["s"])
    block.packed_product(made["q"], made["s"], W, W_scale, made["y"])
    block.top(made["y"], made["index"], made["value"], rest=made["rest"], temperature=temperature)
    block.distill(z, made["index"], made["value"], made["loss"], made["dz"], rest=made["rest"], temperature=temperature)


def room(L, rows, width, columns, k, dtype):
    (q, s) = L.packed_shapes(rows, width)
    new = lambda t, *shape: torch.zeros(shape, dtype=t, device="cuda")  # noqa: E731
    return {"q": new(torch.float8_e4m3fn, *q), "s": new(torch.uint8, *s), "y": new(dtype, rows, columns), "index": new(torch.int32, rows, k),
            "value": new(torch.float32, rows, k), "rest": new(torch.float32, rows), "loss": new(torch.float32, rows),
            "dz": new(dtype, rows, columns)}


def same(a, b):
    return all(torch.equal(a[n].contiguous().view(torch.uint8), b[n].contiguous().view(torch.uint8)) for n in a)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("rows", [3, 150])
def test_a_run_of_them(L, blocks, mode, rows):
    """Every step from what the one before stored, against its definition."""
    width, columns, k, d = 300, 1111, 16, R.DTYPES[mode]
    x, z = noise(1, rows, width).to(d).cuda(), noise(2, rows, columns, std=2.0).to(d).cuda()
    weights = noise(3, columns, width, std=4 / math.sqrt(width)).to(d).cuda()
    W, W_scale = packed(L, blocks, mode, weights)
    made = room(L, rows, width, columns, k, d)
    chain(blocks[mode], x, W, W_scale, k, z, made)
    torch.cuda.synchronize()
    q, s = R.quantise(x.double())
    assert torch.equal(made["q"].view(torch.uint8).cpu(), q) and torch.equal(made["s"].cpu(), s)
    want, off = R.product(R.values(q, s), R.values(W, W_scale), mode)
    assert bool(((made["y"].double().cpu() - want).abs() <= off).all())
    index, value, rest = R.top(made["y"], k, 2.0)
    assert torch.equal(made["index"].cpu(), index) and torch.equal(made["value"].double().cpu(), value)
    assert torch.allclose(made["rest"].double().cpu(), rest, rtol=0, atol=400 * R.U * 20)
    check_distill(blocks[mode], mode, z, index, value.float(), made["rest"].cpu(), 2.0)


def test_streams_at_once(L, blocks):
    """Calls on one block by two streams that overlap: none has a workspace that the other could be in."""
    d, rows, width, columns, k = torch.bfloat16, 200, 512, 9000, 32
    W, W_scale = packed(L, blocks, "bf16", noise(3, columns, width, std=0.1).to(d).cuda())
    inputs = [(noise(i, rows, width).to(d).cuda(), noise(i + 9, rows, columns, std=2.0).to(d).cuda()) for i in range(2)]
    eager = []
    for x, z in inputs:
        eager.append(room(L, rows, width, columns, k, d))
        chain(blocks["bf16"], x, W, W_scale, k, z, eager[-1])
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in inputs], [room(L, rows, width, columns, k, d) for _ in inputs]
    torch.cuda.synchronize()
    for _ in range(3):
        for (x, z), stream, made in zip(inputs, streams, got):
            with torch.cuda.stream(stream):
                chain(blocks["bf16"], x, W, W_scale, k, z, made)
    torch.cuda.synchronize()
    assert same(eager[0], got[0]) and same(eager[1], got[1])


def test_captured_and_replayed(L, blocks):
    d, rows, width, columns, k = torch.float16, 9, 384, 40000, 20
    W, W_scale = packed(L, blocks, "f16", noise(3, columns, width, std=0.1).to(d).cuda())
    x, z = torch.zeros(rows, width, dtype=d, device="cuda"), torch.zeros(rows, columns, dtype=d, device="cuda")
    made = room(L, rows, width, columns, k, d)
    inputs = [(noise(i, rows, width).to(d).cuda(), noise(i + 9, rows, columns, std=2.0).to(d).cuda()) for i in range(3)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain(blocks["f16"], x, W, W_scale, k, z, made)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(blocks["f16"], x, W, W_scale, k, z, made)
    for new_x, new_z in inputs + inputs[:1]:
        x.copy_(new_x)
        z.copy_(new_z)
        graph.replay()
        torch.cuda.synchronize()
        eager = room(L, rows, width, columns, k, d)
        chain(blocks["f16"], new_x, W, W_scale, k, new_z, eager)
        torch.cuda.synchronize()
        assert same(eager, made)


def test_no_rows_are_nothing_to_do(blocks):
    block, d = blocks["bf16"], torch.bfloat16
    new = lambda *shape, dtype=d: torch.zeros(shape, dtype=dtype, device="cuda")  # noqa: E731
    block.quantise(new(0, 5), new(0, 128, dtype=torch.uint8), new(0, 4, dtype=torch.uint8))
    block.packed_product(new(0, 128, dtype=torch.uint8), new(0, 4, dtype=torch.uint8), new(3, 128, dtype=torch.uint8), new(3, 4, dtype=torch.uint8), new(0, 3))
    block.top(new(0, 9), new(0, 2, dtype=torch.int32), new(0, 2, dtype=torch.float32))
    block.distill(new(0, 9), new(0, 2, dtype=torch.int32), new(0, 2, dtype=torch.float32), new(0, dtype=torch.float32), None)
    torch.cuda.synchronize()


# ------------------------------------------------------------------ refusals
@pytest.mark.parametrize("stream", [False, True])
def test_tensors_that_are_refused(L, blocks, stream):
    """By the native hand-over, which leaves them to the checks in Python, and by these directly (a stream is named)."""
    block, d = blocks["bf16"], torch.bfloat16
    more = {"stream": torch.cuda.current_stream()} if stream else {}
    new = lambda *shape, dtype=d, device="cuda": torch.zeros(shape, dtype=dtype, device=device)  # noqa: E731
    u8, i32, f32 = torch.uint8, torch.int32, torch.float32
    x, q, s = new(4, 300), new(4, 384, dtype=u8), new(4, 4, dtype=u8)
    W, Ws, y = new(6, 384, dtype=u8), new(6, 4, dtype=u8), new(4, 6)
    for bad in ((x.float(), q, s), (x.cpu(), q, s), (x.t(), q, s), (x, q[:, :256], s), (x, q[:3], s), (x, q, new(4, 3, dtype=u8)),
                (x, new(4, 768, dtype=u8)[:, :384], s), (x, q.int(), s), (x, q.cpu(), s), (x, q, s.int()), (x[0], q, s)):
        with pytest.raises(ValueError):
            block.quantise(*bad, **more)
    for bad in ((q, s, W[:, :256], Ws, y), (q, s, W, s, y), (q, s, W, Ws, y[:3]), (q, s, W, Ws, y.float()), (q, s, W, Ws, new(6, 4).t()),
                (q[:, :100], s, W[:, :100], Ws, y), (q.cpu(), s, W, Ws, y)):
        with pytest.raises(ValueError):
            block.packed_product(*bad, **more)
    z, index, value, rest = new(4, 50), new(4, 3, dtype=i32), new(4, 3, dtype=f32), new(4, dtype=f32)
    for bad in ((z.float(), index, value), (z, index.long(), value), (z, index, value.half()), (z, index[:3], value), (z, index, value[:, :2]),
                (z, new(3, 4, dtype=i32).t(), value), (z, index.cpu(), value), (z[0], index, value)):
        with pytest.raises(ValueError):
            block.top(*bad, **more)
    with pytest.raises(ValueError):
        block.top(z, index, value, rest=rest[:3], **more)
    loss, dz = new(4, dtype=f32), new(4, 50)
    for bad in ((z, index, value, loss[:2], dz), (z, index, value, loss.half(), dz), (z, index, value, loss, dz[:, :49]), (z, index, value, loss, dz.float()),
                (z, index.long(), value, loss, dz), (z, index, value.cpu(), loss, dz)):
        with pytest.raises(ValueError):
            block.distill(*bad, **more)
    for named in ({"rest": rest[:1]}, {"weight": rest.half()}):
        with pytest.raises(ValueError):
            block.distill(z, index, value, loss, dz, **named, **more)
    for refused in (lambda: block.top(z, new(4, 129, dtype=i32), new(4, 129, dtype=f32), **more), lambda: block.top(z, index, value, temperature=0.0, **more),
                    lambda: block.top(z, index, value, temperature=math.nan, **more), lambda: block.distill(z, index, value, None, None, **more),
                    lambda: block.distill(z, index, value, loss, dz, temperature=-1.0, **more), lambda: block.distill(z, index, value, loss, dz, scale=math.inf, **more),
                    lambda: block.distill(z, index, value, loss, dz, temperature=1e-45, **more)):
        with pytest.raises(L.CcdcError):
            refused()


def test_largest_rows(blocks):
    """2^20 columns are taken, one more is refused."""
    block, columns = blocks["f32"], 1 << 20
    z = noise(1, 1, columns).float().cuda()
    check_top(block, z, 5)
    index, value = torch.tensor([[columns - 1, 0]]), torch.tensor([[1.0, 2.0]])
    check_distill(block, "f32", z, index, value, torch.zeros(1), 1.0)
    z = torch.zeros(1, columns + 1, device="cuda")
    one = lambda t: torch.zeros(1, 1, dtype=t, device="cuda")  # noqa: E731
    import paper_1805_01993_amd as L
    for call in (lambda: block.top(z, one(torch.int32), one(torch.float32)),
                 lambda: block.distill(z, one(torch.int32), one(torch.float32), one(torch.float32)[0], None)):
        with pytest.raises(L.CcdcError):
            call()


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("columns", [300, 520, 1000, 2000, 4000, 20000, 50021])
def test_much_wanted_of_rows(blocks, mode, columns):
    """As many as the list may have: of short rows, where many columns reach any bound, and of rows with equal values, which are listed
    by their columns."""
    random = noise(columns, 12, columns)
    coarse = (random * 2).round()
    few = torch.full_like(random, torch.finfo(R.DTYPES[mode]).min)
    few[:, [7, 33, columns - 1]] = random[:, :3]
    last = torch.zeros_like(random)
    last[:, -100:] = 1.0
    for z in (random, coarse, few, last, random * 0.0, -coarse.abs(), random.sort(1).values):
        for k in (33, 49, 65, 97, 128):
            check_top(blocks[mode], z.to(R.DTYPES[mode]).cuda(), k)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("columns", [100, 1000, 9000, 70000])
def test_infinities_among_the_others(blocks, mode, columns):
    """More infinities than the list takes: the others' sum is one; a NaN beside them makes it none."""
    z = noise(3, 5, columns)
    z[0, [3, 50, columns - 1]] = math.inf
    z[1, ::2] = math.inf
    z[2, 5:] = math.inf
    z[3, [3, 50, columns - 1]], z[3, 77] = math.inf, math.nan
    z[4, 4] = math.inf
    for k in (1, 2, 3, 4):
        check_top(blocks[mode], z.to(R.DTYPES[mode]).cuda(), k)


def test_temperatures_of_no_power(blocks):
    """1 / temperature is a number, and times log2(e) not."""
    import paper_1805_01993_amd as L
    block, z = blocks["f32"], torch.zeros(1, 8, device="cuda")
    index, value = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.zeros(1, 1, device="cuda")
    for call in (lambda: block.top(z, index, value, temperature=3.5e-39),
                 lambda: block.distill(z, index, value, value[0], None, temperature=3.5e-39)):
        with pytest.raises(L.CcdcError):
            call()


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("columns", [524288, 524289, 1 << 20])
def test_long_rows(blocks, mode, columns):
    """Rows that are held in part, and those of which none is: more bits of listed columns than leave room for it."""
    z = noise(7, 2, columns).to(R.DTYPES[mode]).cuda()
    index = torch.tensor([[columns - 1, 0, 70001], [131071, 32768, columns - 2]])
    check_distill(blocks[mode], mode, z, index, noise(8, 2, 3), noise(9, 2), 1.5)


@pytest.mark.parametrize("mode", MODES)
def test_products_of_more_than_64_rows_are_the_same_in_any_batch(blocks, mode):
    """An element's sum has one order whatever tile it is in: nodes that have some of the rows make the same bits of them."""
    wide, outputs = 1152, 2100
    x, xs = random_packed(1, 3000, wide)
    w, ws = random_packed(2, outputs, wide)
    whole = torch.zeros(3000, outputs, dtype=R.DTYPES[mode], device="cuda")
    blocks[mode].packed_product(x, xs, w, ws, whole)
    for rows, columns in ((65, outputs), (333, outputs), (1000, outputs), (500, 70), (2999, 1)):
        y = torch.zeros(rows, columns, dtype=R.DTYPES[mode], device="cuda")
        blocks[mode].packed_product(x[:rows], xs[:rows], w[:columns], ws[:columns], y)
        assert torch.equal(y, whole[:rows, :columns]), (rows, columns)
