"""The trained block at the edges of its definition (include/ccdc.h), against 64 bits.  Needs a GPU."""
import numpy as np
import pytest

import block_reference as R
from test_gpu_block import MODES, SEED, L, close, empty, numbers, torch  # noqa: F401  (fixtures among them)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ties", [0.5, 1.5, 2.5, 6552.5, 6553.5, 65534.5])
def test_dropout_at_ties(torch, L, ties):  # noqa: F811
    """A probability half way between two multiples of 2^-16 goes to the even one: in dropout by itself, of the hidden values and
    in a join (whose factors are 65536 / (65536 - thr), exact to a rounding)."""
    p, thr = ties / 65536, int(np.rint(ties))
    d, F, lengths = 40, 4096, [700]
    keep = R.factors(lengths, [0], F, thr / 65536, 9, SEED)
    block = L.ccdc_block(d, F, "f32", dropout_hidden=p, dropout_out=p, layer=4).bind(lengths).upload()
    x = torch.ones(700, F, device="cuda")
    block.dropout(x, x, p, site=9, seed=SEED)
    assert np.array_equal(x.cpu().numpy(), keep.astype(np.float32))

    rng = np.random.default_rng(1)
    x, xv = numbers(torch, "f32", rng, (700, d))
    W_in, iv = numbers(torch, "f32", rng, (2 * F, d), 1 / 6)
    W_out, ov = numbers(torch, "f32", rng, (d, F), 1 / 64)
    y, z = empty(torch, x, 700, d), empty(torch, x, 700, d)
    block.ffn_forward(x, W_in, W_out, y, seed=SEED)
    close("y", y, R.ffn(lengths, xv, iv, ov, None, R.factors(lengths, [0], F, thr / 65536, 8, SEED), "silu", "f32")["y"])
    block.join_forward(x, x, z, None, seed=SEED)
    one = np.ones(d)
    close("z", z, R.join(xv, xv, one, one, one, R.factors(lengths, [0], d, thr / 65536, 9, SEED), 1.0, float(np.float32(1e-6)), False,
                         "f32")["y"])


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("d,F,rows", [(64, 200, 40), (51, 133, 70)])
def test_what_dropout_takes_out_counts_for_nothing_in_the_gradients(torch, L, mode, act, bad, d, F, rows):  # noqa: F811
    """One token whose gradient is no finite number: hidden values that were taken out of it have gradients of zero, so their rows of
    dW_in are what they are with a gradient of zeros there.  Those that were kept are as bad as it."""
    rng = np.random.default_rng(d)
    at = 17
    block = L.ccdc_block(d, F, mode, activation=act, dropout_hidden=0.4, layer=3).bind([rows, 5]).upload()
    x, _ = numbers(torch, mode, rng, (rows + 5, d))
    W_in, _ = numbers(torch, mode, rng, (2 * F, d), 1 / np.sqrt(d))
    W_out, _ = numbers(torch, mode, rng, (d, F), 1 / np.sqrt(F))
    dy, _ = numbers(torch, mode, rng, (rows + 5, d), 0.25)
    y, saved = torch.empty_like(x), torch.empty(block.saved_bytes, dtype=torch.uint8, device="cuda")
    block.ffn_forward(x, W_in, W_out, y, saved=saved, seed=SEED)
    got = []
    for v in (0.0, bad):
        dy[at] = v
        dx, dW_in, dW_out = torch.empty_like(x), empty(torch, x, 2, 2 * F, d), empty(torch, x, 2, d, F)
        block.ffn_backward(x, W_in, W_out, saved, dy, dx, dW_in, dW_out)
        torch.cuda.synchronize()
        assert torch.isfinite(torch.cat((dx[:at], dx[at + 1:])).float()).all()
        got.append(dW_in)
    assert torch.isfinite(got[0].float()).all() and torch.equal(got[0][1], got[1][1])
    out = torch.from_numpy(R.factors([rows, 5], [0, 1], F, float(np.float32(0.4)), 6, SEED)[at] == 0).cuda()
    for half in (0, 1):                                # rows of Wg, of Wu
        zeros, wrong = (g[0, half * F:half * F + F] for g in got)
        assert torch.equal(zeros[out], wrong[out])
        assert not torch.isfinite(wrong[~out].float()).any(1).any()


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_gradients_are_the_same_in_every_batch_with_every_activation(torch, L, mode, act):  # noqa: F811
    """Alone and among files that make the products take larger tiles, which are kernels of their own: the same bits of y, dx and
    the weights' gradients."""
    rng = np.random.default_rng(12)
    d, F, lengths = 264, 2060, [70, 513, 1, 300, 640, 129, 700, 650]
    at = np.concatenate(([0], np.cumsum(lengths)))
    x, _ = numbers(torch, mode, rng, (sum(lengths), d))
    dy, _ = numbers(torch, mode, rng, (sum(lengths), d), 0.1)
    W_in, _ = numbers(torch, mode, rng, (2 * F, d), 1 / 4)
    W_out, _ = numbers(torch, mode, rng, (d, F), 1 / 45)

    def results(files):
        block = L.ccdc_block(d, F, mode, activation=act, dropout_hidden=0.15, layer=1).bind([lengths[n] for n in files], files).upload()
        rows = torch.from_numpy(np.concatenate([np.arange(at[n], at[n + 1]) for n in files])).cuda()
        px, pdy = x[rows].contiguous(), dy[rows].contiguous()
        saved = torch.empty(block.saved_bytes, dtype=torch.uint8, device="cuda")
        y, dx = torch.empty_like(px), torch.empty_like(px)
        dW_in, dW_out = empty(torch, x, len(files), 2 * F, d), empty(torch, x, len(files), d, F)
        block.ffn_forward(px, W_in, W_out, y, saved=saved, seed=SEED)
        block.ffn_backward(px, W_in, W_out, saved, pdy, dx, dW_in, dW_out)
        torch.cuda.synchronize()
        by_file = lambda t: torch.split(t, [lengths[n] for n in files])  # noqa: E731
        return {n: (a, b, dW_in[i], dW_out[i]) for i, (n, a, b) in enumerate(zip(files, by_file(y), by_file(dx)))}

    everything = results(list(range(8)))
    for files in ([5, 0, 2], [3], [4, 6, 1], [7]):
        for n, parts in results(files).items():
            for name, a, b in zip(("y", "dx", "dW_in", "dW_out"), parts, everything[n]):
                assert torch.equal(a, b), f"file {n} in {files}: {name} differs"


# ------------------------------------------------------------------ forms of the calls
@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("d,F,ld", [(64, 96, 64), (72, 101, 72), (51, 96, 51), (51, 133, 57), (64, 96, 67)])
def test_forms_of_the_gradient_call(torch, L, mode, d, F, ld):  # noqa: F811
    """dx in the place of dy, dx alone and the weights' gradients alone: the bits of the whole call, with matrices that the products take
    as they are and that are laid out first, and hidden sizes of whole packs and not."""
    rng = np.random.default_rng(d + F)
    M, N = 83, 3
    block = L.ccdc_block(d, F, mode, dropout_hidden=0.1).bind([50, 0, 33]).upload()
    x, _ = numbers(torch, mode, rng, (M, d), ld=ld)
    dy, _ = numbers(torch, mode, rng, (M, d), 0.25, ld=ld)
    W_in, _ = numbers(torch, mode, rng, (2 * F, d), 1 / 8)
    W_out, _ = numbers(torch, mode, rng, (d, F), 1 / 10)
    saved = torch.empty(block.saved_bytes, dtype=torch.uint8, device="cuda")
    block.ffn_forward(x, W_in, W_out, empty(torch, x, M, d), saved=saved, seed=SEED)
    kept = saved.clone()

    def call(dx, weights=True):
        dW = (empty(torch, x, N, 2 * F, d), empty(torch, x, N, d, F)) if weights else (None, None)
        block.ffn_backward(x, W_in, W_out, saved, dy, dx, *dW)
        torch.cuda.synchronize()
        return (dx,) + dW

    want = call(empty(torch, x, M, d))
    assert all(torch.isfinite(t.float()).all() for t in want)
    assert torch.equal(call(empty(torch, x, M, d, ld=ld + 3), weights=False)[0], want[0])
    assert all(torch.equal(a, b) for a, b in zip(call(None)[1:], want[1:]))
    assert all(torch.equal(a, b) for a, b in zip(call(dy), want))              # last: dy is gone
    assert torch.equal(saved, kept)                                            # only read


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("rows", [1, 4, 7, 16, 24, 33, 64])
@pytest.mark.parametrize("d,F", [(256, 320), (99, 203)])
def test_few_rows_with_dropout(torch, L, mode, act, rows, d, F):  # noqa: F811
    """The kernels for few rows, which make an element's factor by itself: rows of several files, numbers of their own."""
    rng = np.random.default_rng(rows)
    lengths, ids = [rows // 2, 0, rows - rows // 2], [11, 3, 1 << 30]
    block = L.ccdc_block(d, F, mode, activation=act, dropout_hidden=0.3, layer=6).bind(lengths, ids).upload()
    x, xv = numbers(torch, mode, rng, (rows, d), ld=d + 5)
    W_in, iv = numbers(torch, mode, rng, (2 * F, d), 1 / np.sqrt(d))
    W_out, ov = numbers(torch, mode, rng, (d, F), 1 / np.sqrt(F))
    y = empty(torch, x, rows, d, ld=d + 2)
    block.ffn_forward(x, W_in, W_out, y, seed=SEED)
    keep = R.factors(lengths, ids, F, float(np.float32(0.3)), 12, SEED)
    close("y", y, R.ffn(lengths, xv, iv, ov, None, keep, act, mode)["y"])


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("rows,d,F", [(65, 264, 2060), (130, 72, 4096), (66, 9, 5000)])
def test_second_products_in_ranges_into_rows_of_any_stride(torch, L, mode, rows, d, F):  # noqa: F811
    rng = np.random.default_rng(rows)
    block = L.ccdc_block(d, F, mode, dropout_hidden=0.2, layer=6).bind([rows]).upload()
    x, xv = numbers(torch, mode, rng, (rows, d))
    W_in, iv = numbers(torch, mode, rng, (2 * F, d), 1 / np.sqrt(d))
    W_out, ov = numbers(torch, mode, rng, (d, F), 1 / np.sqrt(F))
    room = torch.full((rows, d + 13), float("nan"), dtype=x.dtype, device="cuda")
    block.ffn_forward(x, W_in, W_out, room[:, 3:3 + d], seed=SEED)
    keep = R.factors([rows], [0], F, float(np.float32(0.2)), 12, SEED)
    close("y", room[:, 3:3 + d], R.ffn([rows], xv, iv, ov, None, keep, "silu", mode)["y"])
    assert torch.isnan(room[:, :3].float()).all() and torch.isnan(room[:, 3 + d:].float()).all()


# ------------------------------------------------------------------ infinities and what is no number
BAD = [float("inf"), float("-inf"), float("nan")]


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("rows,d,F", [(1, 64, 96), (3, 200, 136), (8, 99, 203), (16, 64, 96), (40, 256, 320), (64, 99, 203), (90, 72, 1100),
                                      (300, 51, 133)])
def test_a_row_that_is_no_number_leaves_the_others_alone(torch, L, mode, bad, rows, d, F):  # noqa: F811
    """One bad input spoils its token's outputs and no other token's, in the kernels of every number of rows; one bad element of W_out
    spoils its column."""
    rng = np.random.default_rng(rows)
    block = L.ccdc_block(d, F, mode).bind([rows]).upload()
    x, _ = numbers(torch, mode, rng, (rows, d))
    W_in, _ = numbers(torch, mode, rng, (2 * F, d), 1 / np.sqrt(d))
    W_out, _ = numbers(torch, mode, rng, (d, F), 1 / np.sqrt(F))
    at, column = rows // 2, d - 1
    y, spoilt = empty(torch, x, rows, d), empty(torch, x, rows, d)
    block.ffn_forward(x, W_in, W_out, y)
    assert torch.isfinite(y.float()).all()
    x2 = x.clone()
    x2[at, column] = bad
    block.ffn_forward(x2, W_in, W_out, spoilt)
    others = torch.arange(rows, device="cuda") != at
    assert torch.equal(spoilt[others], y[others]) and not torch.isfinite(spoilt[at].float()).any()
    W2 = W_out.clone()
    W2[column, F - 1] = bad
    spoilt = empty(torch, x, rows, d)
    block.ffn_forward(x, W_in, W2, spoilt)
    assert torch.equal(spoilt[:, :column], y[:, :column])
    assert not torch.isfinite(spoilt[:, column].float()).all()
    if mode == "f32":                                  # documented: of an infinite operand the products make no number
        assert torch.isnan(spoilt[:, column]).any()


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("lengths,d,F", [([20, 3, 0, 41], 72, 104), ([20, 3, 0, 41], 51, 133), ([700, 650, 90], 264, 2060)])
def test_a_file_that_is_no_number_leaves_the_others_alone(torch, L, mode, bad, lengths, d, F):  # noqa: F811
    """One bad token of a file: the other files' gradients keep their bits, and so do the other tokens'."""
    rng = np.random.default_rng(d)
    M, N, spoilt = sum(lengths), len(lengths), 1
    at = lengths[0] + lengths[1] - 1                   # the last of the second file
    block = L.ccdc_block(d, F, mode).bind(lengths).upload()
    x, _ = numbers(torch, mode, rng, (M, d))
    dy, _ = numbers(torch, mode, rng, (M, d), 0.25)
    W_in, _ = numbers(torch, mode, rng, (2 * F, d), 1 / np.sqrt(d))
    W_out, _ = numbers(torch, mode, rng, (d, F), 1 / np.sqrt(F))
    results = []
    for v in (None, bad):
        if v is not None:
            x[at, 0] = v
        saved = torch.empty(block.saved_bytes, dtype=torch.uint8, device="cuda")
        y, dx, dW_in, dW_out = empty(torch, x, M, d), empty(torch, x, M, d), empty(torch, x, N, 2 * F, d), empty(torch, x, N, d, F)
        block.ffn_forward(x, W_in, W_out, y, saved=saved)
        block.ffn_backward(x, W_in, W_out, saved, dy, dx, dW_in, dW_out)
        torch.cuda.synchronize()
        results.append((y, dx, dW_in, dW_out))
    rows, files = torch.arange(M, device="cuda") != at, torch.arange(N, device="cuda") != spoilt
    for i, (good, wrong) in enumerate(zip(*results)):
        same = files if i > 1 else rows
        assert torch.isfinite(good.float()).all()
        assert torch.equal(good[same], wrong[same]) and not torch.isfinite(wrong[~same].float()).all()


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("centred", [False, True])
@pytest.mark.parametrize("d", [7, 520, 1500, 3001, 9000])
def test_a_row_of_a_join_that_is_no_number_leaves_the_others_alone(torch, L, mode, bad, centred, d):  # noqa: F811
    """Rows share wavefronts and barriers, and files their sums, with others: those keep their bits."""
    rng = np.random.default_rng(d)
    lengths = [5, 40, 0, 3]
    M, N, at = 48, 4, 44                               # the last row of the second file
    block = L.ccdc_block(d, 8, mode, norm="centred" if centred else "rms", dropout_out=0.1).bind(lengths).upload()
    x, f, dn, dr = (numbers(torch, mode, rng, (M, d))[0] for _ in range(4))
    rows, files = torch.arange(M, device="cuda") != at, torch.arange(N, device="cuda") != 1
    results = []
    for v in (None, bad):
        if v is not None:
            x[at, d - 1] = f[at, 0] = dn[at, 0] = v
        y, n, dx, df = (empty(torch, x, M, d) for _ in range(4))
        sums = [empty(torch, x, N, d) for _ in range(3)]
        block.join_forward(x, f, y, n, seed=SEED)
        block.join_backward(dn, dr, y, f, dx, df, dw_post=sums[0], dgate=sums[1], dw_pre=sums[2], seed=SEED)
        torch.cuda.synchronize()
        results.append([y, n, dx, df] + sums)
    for i, (good, wrong) in enumerate(zip(*results)):
        same = files if i > 3 else rows
        assert torch.isfinite(good.float()).all()
        assert torch.equal(good[same], wrong[same]) and not torch.isfinite(wrong[~same].float()).all()
