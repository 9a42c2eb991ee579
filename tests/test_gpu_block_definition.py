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
