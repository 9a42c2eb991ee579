"""The sums over a row of a join and of its gradient, at every width, with bounds that do not grow with it, and rows whose last column or
last pack of columns has most of what is summed: a sum that leaves out any of it shows.  The kernels need a GPU; that the bounds
notice does not.

A lane adds at most 16 elements (fused, one rounding each), a wavefront its 64 lanes in 6 steps, a workgroup at most 16
wavefronts one after the other: a term is rounded at most 40 times with what follows (division, eps, root, reciprocal: 5, of which
the sum's count half), where terms cancel relative to the sum of their magnitudes.  With the products before (a weight, a
gate, a factor of dropout) that is within E = 64 x 2^-24.  Where the mean is subtracted its own error is as large against the mean of
magnitudes, which `scale` has; in the squares it cancels to second order."""
import numpy as np
import pytest

import block_reference as R
from test_gpu_block import MODES, SEED, L, close, empty, numbers, torch  # noqa: F401  (fixtures among them)

E = 64 * 2.0 ** -24
WIDTHS = [1, 7, 64, 513, 1000, 2041, 4096, 5003, 8192, 12001, 16384]
LENGTHS = [3, 0, 34, 1]
EPS, RHO = float(np.float32(1e-5)), 0.75


def normed(v, centred, seen):
    """R.normed with statistics of the first `seen` columns only (planted), and what bounds its error: the magnitudes it comes of."""
    d, part = v.shape[1], v[:, :seen]
    mean = part.sum(1, keepdims=True) / d if centred else 0.0
    rstd = 1 / np.sqrt((np.square(part - mean)).sum(1, keepdims=True) / d + EPS)
    return (v - mean) * rstd, rstd, (np.abs(v) + (np.abs(v).mean(1, keepdims=True) if centred else 0)) * rstd


def join(x, f, w_post, gate, w_pre, keep, centred, mode, seen):
    """{name: (value, bound)}"""
    u, tiny, A = R.ROUND[mode], R.TINY[mode], np.abs
    hat, _, scale = normed(f, centred, seen)
    y = RHO * x + gate * keep * (hat * w_post)
    B = 2 * E * (A(RHO * x) + A(gate * keep * w_post) * scale)
    out = {"y": (y, B + u * A(y) + tiny)}
    hat, rstd, scale = normed(y, centred, seen)
    n = hat * w_pre
    # n follows y by at most rstd, its row's mean and norm by the mean of y's errors
    Bn = A(w_pre) * (rstd * (B + B.mean(1, keepdims=True) + A(hat) * np.sqrt((B * B).mean(1, keepdims=True))) + 2 * E * scale)
    out["n"] = n, Bn + u * A(n) + tiny
    return out


def norm_gradient(e, hat, rstd, centred, seen):
    d = e.shape[1]
    g = e - hat * (e * hat)[:, :seen].sum(1, keepdims=True) / d
    return rstd * (g - e[:, :seen].sum(1, keepdims=True) / d if centred else g)


def size_of(e, scale, rstd, centred):
    """The magnitudes that such a gradient comes of."""
    return rstd * (e + scale * (e * scale).mean(1, keepdims=True) + (e.mean(1, keepdims=True) if centred else 0))


def join_gradient(dn, dr, y, f, w_post, gate, w_pre, keep, centred, mode, seen):
    u, tiny, A = R.ROUND[mode], R.TINY[mode], np.abs
    hat, rstd, scale = normed(y, centred, seen)
    dy = dr + norm_gradient(dn * w_pre, hat, rstd, centred, seen)
    B = E * A(dr) + 4 * E * size_of(A(dn * w_pre), scale, rstd, centred)
    out = {"dx": (RHO * dy, RHO * B + u * A(RHO * dy) + E * A(dy) + tiny)}
    hat, rstd, scale = normed(f, centred, seen)
    w = gate * w_post
    df = norm_gradient(keep * dy * w, hat, rstd, centred, seen)
    out["df"] = df, 4 * E * size_of(keep * A(dy) * A(w), scale, rstd, centred) + size_of(keep * B * A(w), scale, rstd, centred) + u * A(df) + tiny
    return out


def rows(d, where, rng):
    """x, f, dn, dr in 32 bits: even, or with 94 % of a row's squares in its last column or its last pack of eight."""
    M = sum(LENGTHS)
    out = [rng.normal(mean, std, (M, d)).astype(np.float32) for mean, std in ((0, 2.0), (0.3, 0.5), (0, 0.3), (0, 0.2))]
    if where != "even":
        last = 1 if where == "column" else (d - 1) % 8 + 1
        for t in out:
            t[:, d - last:] *= 4 * np.sqrt(d / last)
    return out


def parameters(d, rng):
    """w_post, gate, w_pre"""
    return [rng.normal(mean, std, d).astype(np.float32) for mean, std in ((1.0, 0.2), (0.5, 0.3), (1.0, 0.2))]


@pytest.mark.parametrize("d", [w for w in WIDTHS if w >= 64])
@pytest.mark.parametrize("centred", [False, True])
@pytest.mark.parametrize("where", ["even", "column", "pack"])
def test_bounds_notice_what_sums_leave_out(d, centred, where):
    """Statistics that leave out the last column (where it has most), or the last pack, are past the bounds."""
    rng = np.random.default_rng(d)
    x, f, dn, dr = (t.astype(float) for t in rows(d, where, rng))
    w_post, gate, w_pre = (t.astype(float) for t in parameters(d, rng))
    one = np.ones_like(x)
    out_of = 1 if where == "column" else (d - 1) % 8 + 1
    right = join(x, f, w_post, gate, w_pre, one, centred, "f32", d)
    wrong = join(x, f, w_post, gate, w_pre, one, centred, "f32", d - out_of)
    y = right["y"][0]
    right |= join_gradient(dn, dr, y, f, w_post, gate, w_pre, one, centred, "f32", d)
    wrong |= join_gradient(dn, dr, y, f, w_post, gate, w_pre, one, centred, "f32", d - out_of)
    for name in right:
        off = np.abs(wrong[name][0] - right[name][0]) / right[name][1]
        assert off.max() > 2, f"{name}: {off.max():.2g} of the bound"


@pytest.mark.gpu
@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("centred", [False, True])
@pytest.mark.parametrize("where", ["even", "column", "pack"])
def test_sums_over_a_row(torch, L, mode, d, centred, where):  # noqa: F811
    rng = np.random.default_rng(d)
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[mode]
    t = [torch.from_numpy(v).to(dtype) for v in rows(d, where, rng) + parameters(d, rng)]
    x, f, dn, dr, w_post, gate, w_pre = (v.cuda() for v in t)
    v = [a.double().numpy() for a in t]
    block = L.ccdc_block(d, 8, mode, norm="centred" if centred else "rms", eps=EPS, residual_scale=RHO, dropout_out=0.25,
                         layer=2).bind(LENGTHS).upload()
    keep = R.factors(LENGTHS, range(len(LENGTHS)), d, 0.25, 5, SEED)
    y, n, dx, df = (empty(torch, x, *x.shape) for _ in range(4))
    names = dict(w_post=w_post, gate=gate, w_pre=w_pre, seed=SEED)
    block.join_forward(x, f, y, n, **names)
    block.join_backward(dn, dr, y, f, dx, df, **names)
    torch.cuda.synchronize()
    want = join(v[0], v[1], v[4], v[5], v[6], keep, centred, mode, d)
    want |= join_gradient(v[2], v[3], y.double().cpu().numpy(), v[1], v[4], v[5], v[6], keep, centred, mode, d)
    for name, got in (("y", y), ("n", n), ("dx", dx), ("df", df)):
        close(name, got, want[name])
