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
