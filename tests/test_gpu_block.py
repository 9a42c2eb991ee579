"""The trained block on the GPU against its definition in 64 bits, element by element, within bounds that follow from the
roundings alone (block_reference.py): feed-forward, joins and dropout with their gradients, over types, odd sizes, strides, files of
no and of one token, and the block in front of the shuffle.  Needs a GPU."""
import numpy as np
import pytest

import block_reference as R

pytestmark = pytest.mark.gpu

MODES = ["bf16", "f16", "f32"]
SEED = 0x9E3779B97F4A7C15


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    torch.cuda.set_device(0)
    return torch


@pytest.fixture(scope="module")
def L(torch):
    import paper_1805_01993_amd as lib
    lib.load_library()
    return lib


def numbers(torch, mode, rng, shape, std=1.0, mean=0.0, ld=None, shift=0):
    """A tensor of the mode's type and its values in 64 bits; ld: row stride, shift: elements into its allocation."""
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[mode]
    t = torch.from_numpy(rng.normal(mean, std, shape).astype(np.float32)).to(dtype)
    values = t.double().numpy()
    if ld is None and not shift:
        return t.cuda(), values
    rows, columns = shape
    ld = columns if ld is None else ld
    room = torch.full((shift + rows * ld + 64,), float("nan"), dtype=dtype, device="cuda")
    view = room[shift:].as_strided((rows, columns), (ld, 1), storage_offset=shift)
    view.copy_(t.cuda())
    return view, values


def empty(torch, like, *shape, ld=None):
    """A result's room, full of NaN; ld: row stride."""
    if ld is None:
        return torch.full(shape, float("nan"), dtype=like.dtype, device="cuda")
    return torch.full((shape[0] * ld + 8,), float("nan"), dtype=like.dtype, device="cuda").as_strided(shape, (ld, 1))


def close(name, got, want):
    value, bound = want
    got = got.double().cpu().numpy()
    assert got.shape == value.shape, f"{name}: {got.shape} and {value.shape}"
    assert np.isfinite(got).all(), f"{name}: {(~np.isfinite(got)).sum()} values are not finite"
    off = np.abs(got - value) / bound
    assert off.size == 0 or off.max() <= 1, f"{name}: {off.max():.3g} times the bound at {np.unravel_index(off.argmax(), off.shape)}"


# ------------------------------------------------------------------ feed-forward
def run_ffn(torch, L, lengths, d, F, mode, act="silu", p=0.0, ids=None, train=True, ldx=None, shift=0, room=0):
    rng = np.random.default_rng(len(lengths) * 1000 + d + F)
    M, ids = sum(lengths), list(range(len(lengths))) if ids is None else ids
    block = L.ccdc_block(d, F, mode, activation=act, dropout_hidden=p, layer=5).bind(lengths, ids).upload()
    x, xv = numbers(torch, mode, rng, (M, d), ld=ldx, shift=shift)
    W_in, iv = numbers(torch, mode, rng, (2 * F, d), 1 / np.sqrt(d))
    W_out, ov = numbers(torch, mode, rng, (d, F), 1 / np.sqrt(F))
    dy, gv = numbers(torch, mode, rng, (M, d), 0.25, ld=ldx, shift=shift)
    keep = R.factors(lengths, ids, F, float(np.float32(p)), 10, SEED) if p else np.ones((M, F))
    want = R.ffn(lengths, xv, iv, ov, gv if train else None, keep, act, mode)
    y = empty(torch, x, M, d, ld=ldx)
    if not train:
        block.ffn_forward(x, W_in, W_out, y, seed=SEED)
        return {"y": y}, want
    saved = torch.full((block.saved_bytes,), 255, dtype=torch.uint8, device="cuda")
    dx = empty(torch, x, M, d, ld=ldx)
    V = empty(torch, x, len(lengths), 3 * F * d + room)
    dW_in, dW_out = V[:, :2 * F * d].unflatten(1, (2 * F, d)), V[:, 2 * F * d:3 * F * d].unflatten(1, (d, F))
    block.ffn_forward(x, W_in, W_out, y, saved=saved, seed=SEED)
    block.ffn_backward(x, W_in, W_out, saved, dy, dx, dW_in, dW_out)
    torch.cuda.synchronize()
    if room:
        assert torch.isnan(V[:, 3 * F * d:].float()).all(), "written past a file's gradients"
    block.close()
    return {"y": y, "dx": dx, "dW_in": dW_in, "dW_out": dW_out}, want


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("lengths,d,F", [
    ([1], 8, 8), ([1], 1, 1), ([3], 5, 3), ([7], 64, 64), ([65], 128, 200), ([130], 72, 136),
    ([0, 5, 1, 0, 64, 130, 0], 136, 120),          # files of no token, first and last among them
    ([33, 31, 64], 515, 133),                      # whole packs of nothing
    ([300], 264, 392), ([257, 1], 130, 1030)])
def test_ffn_training(torch, L, mode, lengths, d, F):
    got, want = run_ffn(torch, L, lengths, d, F, mode)
    for name in got:
        close(name, got[name], want[name])


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("act", ["gelu", "relu", "silu"])
def test_ffn_activations_with_dropout(torch, L, mode, act):
    got, want = run_ffn(torch, L, [40, 0, 29], 96, 141, mode, act, p=0.3, ids=[7, 2, 1 << 30])
    for name in got:
        close(name, got[name], want[name])


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("ldx,shift", [(200, 0), (201, 0), (200, 3), (195, 1)])
def test_ffn_strides_and_alignment(torch, L, mode, ldx, shift):
    got, want = run_ffn(torch, L, [50, 21], 192, 96, mode, ldx=ldx, shift=shift, room=5)
    for name in got:
        close(name, got[name], want[name])


def test_ffn_rows_far_apart(torch, L):
    """Row strides with which 64 rows are over 2^32 bytes: columns of a matrix of 34 million."""
    got, want = run_ffn(torch, L, [50, 20], 64, 72, "bf16", ldx=(1 << 25) + 8)
    for name in got:
        close(name, got[name].contiguous(), want[name])
    got, want = run_ffn(torch, L, [9], 64, 72, "bf16", train=False, ldx=(1 << 25) + 8)
    close("y", got["y"].contiguous(), want["y"])


@pytest.mark.parametrize("mode", MODES)
def test_ffn_everything_dropped(torch, L, mode):
    got, want = run_ffn(torch, L, [9], 32, 48, mode, p=1.0)
    for name in got:
        assert (got[name] == 0).all(), name


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("rows", [1, 2, 5, 9, 16, 17, 33, 64, 65, 100])
@pytest.mark.parametrize("d,F", [(512, 640), (203, 411)])
def test_ffn_few_rows(torch, L, mode, rows, d, F):
    got, want = run_ffn(torch, L, [rows], d, F, mode, "gelu", train=False)
    close("y", got["y"], want["y"])


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("rows,d,F", [(65, 264, 2060), (130, 72, 4096), (300, 515, 1333), (129, 1000, 1536), (66, 9, 5000)])
def test_ffn_rows_that_leave_the_chip_without_work(torch, L, mode, rows, d, F):
    """The second product in ranges of its k, whole and not, that are added up."""
    got, want = run_ffn(torch, L, [rows], d, F, mode, train=False)
    close("y", got["y"], want["y"])


@pytest.mark.parametrize("mode", MODES)
def test_ffn_large_tiles(torch, L, mode):
    """Enough tiles of 256 x 256 for those kernels, sizes that end inside one."""
    got, want = run_ffn(torch, L, [1100, 0, 963], 1048, 3992, mode, p=0.1)
    for name in got:
        close(name, got[name], want[name])


@pytest.mark.parametrize("mode", MODES)
def test_ffn_rows_of_a_larger_batch(torch, L, mode):
    """Fewer rows than the batch is bound to: the same values, nothing behind them written."""
    rng = np.random.default_rng(3)
    d, F = 256, 320
    block = L.ccdc_block(d, F, mode).bind([300]).upload()
    x, xv = numbers(torch, mode, rng, (300, d))
    W_in, iv = numbers(torch, mode, rng, (2 * F, d), 1 / 16)
    W_out, ov = numbers(torch, mode, rng, (d, F), 1 / 16)
    for rows in (0, 1, 40, 299):
        y = empty(torch, x, 300, d)
        block.ffn_forward(x[:rows], W_in, W_out, y[:rows])
        torch.cuda.synchronize()
        assert torch.isnan(y[rows:].float()).all()
        if rows:
            want = R.ffn([rows], xv[:rows], iv, ov, None, np.ones((rows, F)), "silu", mode)
            close("y", y[:rows], want["y"])


@pytest.mark.parametrize("mode", MODES)
def test_a_files_gradients_are_the_same_in_every_batch(torch, L, mode):
    """What a receiver cancels it has computed itself: bit for bit, on its own files in an order of its own, with tiles of another size."""
    rng = np.random.default_rng(11)
    d, F, lengths = 264, 2060, [70, 513, 1, 300, 640, 129, 700, 650]
    at = np.concatenate(([0], np.cumsum(lengths)))
    x, _ = numbers(torch, mode, rng, (sum(lengths), d))
    dy, _ = numbers(torch, mode, rng, (sum(lengths), d), 0.1)
    W_in, _ = numbers(torch, mode, rng, (2 * F, d), 1 / 16)
    W_out, _ = numbers(torch, mode, rng, (d, F), 1 / 45)
    w_post, _ = numbers(torch, mode, rng, (d,))
    w_pre, _ = numbers(torch, mode, rng, (d,))
    gate, _ = numbers(torch, mode, rng, (d,))

    def gradients(files):
        block = L.ccdc_block(d, F, mode, dropout_hidden=0.1, dropout_out=0.2, layer=1).bind([lengths[n] for n in files], files).upload()
        rows = np.concatenate([np.arange(at[n], at[n + 1]) for n in files])
        part = lambda t: t[torch.from_numpy(rows).cuda()].contiguous()  # noqa: E731
        px, pdy = part(x), part(dy)
        saved = torch.empty(block.saved_bytes, dtype=torch.uint8, device="cuda")
        y, dx = torch.empty_like(px), torch.empty_like(px)
        dW_in, dW_out = empty(torch, x, len(files), 2 * F, d), empty(torch, x, len(files), d, F)
        block.ffn_forward(px, W_in, W_out, y, saved=saved, seed=SEED)
        block.ffn_backward(px, W_in, W_out, saved, pdy, dx, dW_in, dW_out)
        z, n, df = torch.empty_like(px), torch.empty_like(px), torch.empty_like(px)
        sums = [empty(torch, x, len(files), d) for _ in range(3)]
        names = dict(w_post=w_post, gate=gate, w_pre=w_pre, seed=SEED)
        block.join_forward(px, y, z, n, **names)
        block.join_backward(pdy, pdy, z, y, dx, df, dw_post=sums[0], dgate=sums[1], dw_pre=sums[2], **names)
        torch.cuda.synchronize()
        return {n: [t[i] for t in [dW_in, dW_out] + sums] for i, n in enumerate(files)}

    everything = gradients(list(range(8)))
    for files in ([5, 0, 2], [3], [4, 6, 1]):
        for n, parts in gradients(files).items():
            for i, (a, b) in enumerate(zip(parts, everything[n])):
                assert torch.equal(a, b), f"file {n} in {files}: gradient {i} differs"


@pytest.mark.parametrize("mode", MODES)
def test_a_batch_without_tokens(torch, L, mode):
    """Files, but no token in any: nothing to compute, and gradients of zeros."""
    d, F = 24, 40
    block = L.ccdc_block(d, F, mode).bind([0, 0, 0]).upload()
    new = lambda *s: torch.full(s, float("nan"), dtype=block.dtype, device="cuda")  # noqa: E731
    none, W_in, W_out, w = new(0, d), new(2 * F, d).zero_(), new(d, F).zero_(), new(d).zero_()
    saved = torch.empty(block.saved_bytes, dtype=torch.uint8, device="cuda")
    dW_in, dW_out, sums = new(3, 2 * F, d), new(3, d, F), [new(3, d) for _ in range(3)]
    block.ffn_forward(none, W_in, W_out, none, saved=saved)
    block.ffn_backward(none, W_in, W_out, saved, none, none, dW_in, dW_out)
    block.join_forward(none, none, none, none, w_post=w, gate=w, w_pre=w)
    block.join_backward(none, none, none, none, none, none, w_post=w, gate=w, w_pre=w, dw_post=sums[0], dgate=sums[1], dw_pre=sums[2])
    block.dropout(none, none, 0.5, site=0)
    torch.cuda.synchronize()
    assert all((t == 0).all() for t in [dW_in, dW_out] + sums)


# ------------------------------------------------------------------ joins
def run_join(torch, L, lengths, d, mode, centred=False, p=0.0, gate="shared", parts="xfn", ld=None, parameters=True):
    rng = np.random.default_rng(d + len(lengths))
    M, N, ids = sum(lengths), len(lengths), [3 * n + 1 for n in range(len(lengths))]
    block = L.ccdc_block(d, 8, mode, norm="centred" if centred else "rms", eps=1e-5, residual_scale=0.75, dropout_out=p,
                         layer=2).bind(lengths, ids).upload()
    x, xv = numbers(torch, mode, rng, (M, d), 2.0, ld=ld)
    f, fv = numbers(torch, mode, rng, (M, d), 0.5, 0.3, ld=ld) if "f" in parts else (None, None)
    w_post, pv = numbers(torch, mode, rng, (d,), 0.2, 1.0) if parameters else (None, np.ones(d))
    w_pre, rv = numbers(torch, mode, rng, (d,), 0.2, 1.0) if parameters else (None, np.ones(d))
    g, gv = {"none": lambda: (None, np.ones(d)), "shared": lambda: numbers(torch, mode, rng, (d,), 0.5),
             "files": lambda: numbers(torch, mode, rng, (N, d), 0.5)}[gate]()
    gv = np.repeat(gv, lengths, 0) if gate == "files" else gv
    keep = R.factors(lengths, ids, d, float(np.float32(p)), 5, SEED) if p else np.ones((M, d))
    names = dict(w_post=w_post, gate=g, w_pre=w_pre, seed=SEED)
    new = lambda: empty(torch, x, M, d, ld=ld)  # noqa: E731
    y, n = new(), new() if "n" in parts else None
    block.join_forward(x, f, y, n, **names)
    torch.cuda.synchronize()
    eps = float(np.float32(1e-5))
    want = R.join(xv, fv, pv, gv, rv, keep, 0.75, eps, centred, mode)
    close("y", y, want["y"])
    if n is not None:
        close("n", n, want["n"])
    dn, dnv = numbers(torch, mode, rng, (M, d), 0.3, ld=ld) if "n" in parts else (None, None)
    dr, drv = numbers(torch, mode, rng, (M, d), 0.2, ld=ld) if "x" in parts else (None, None)
    dx, df = new(), new() if f is not None else None
    rows = empty(torch, x, N, 3 * d + 1)
    sums = {"dw_pre": rows[:, :d] if dn is not None else None, "dw_post": rows[:, d:2 * d] if f is not None else None,
            "dgate": rows[:, 2 * d:3 * d] if f is not None else None}
    block.join_backward(dn, dr, y if dn is not None else None, f, dx, df, **sums, **names)
    torch.cuda.synchronize()
    want = R.join_gradient(lengths, dnv, drv, y.double().cpu().numpy(), fv, pv, gv, rv, keep, 0.75, eps, centred, mode)
    for name, t in {"dx": dx, "df": df, **sums}.items():
        if t is not None:
            close(name, t, want[name])
    assert torch.isnan(rows[:, 3 * d:].float()).all()
    block.close()


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("d", [1, 7, 64, 513, 1000, 2041, 4096, 5003, 8192, 12001, 16384])
@pytest.mark.parametrize("centred", [False, True])
def test_join(torch, L, mode, d, centred):
    run_join(torch, L, [3, 0, 70, 1], d, mode, centred, p=0.2)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("gate", ["none", "shared", "files"])
@pytest.mark.parametrize("parts", ["xfn", "xf", "xn", "fn"])
def test_join_parts(torch, L, mode, gate, parts):
    run_join(torch, L, [0, 33, 65, 2], 520, mode, False, p=0.1, gate=gate, parts=parts, ld=527)


@pytest.mark.parametrize("mode", MODES)
def test_join_without_parameters(torch, L, mode):
    run_join(torch, L, [40], 96, mode, True, gate="none", parameters=False)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("d", [96, 3000, 9000])
def test_join_in_place(torch, L, mode, d):
    rng = np.random.default_rng(1)
    block = L.ccdc_block(d, 8, mode, dropout_out=0.1).bind([21, 12]).upload()
    x, f, dn, dr = (numbers(torch, mode, rng, (33, d))[0] for _ in range(4))
    gate, _ = numbers(torch, mode, rng, (d,))
    y, n, dx, df = (torch.empty_like(x) for _ in range(4))
    block.join_forward(x, f, y, n, gate=gate, seed=1)
    block.join_backward(dn, dr, y, f, dx, df, gate=gate, seed=1)
    for first, second in ((0, 1), (1, 0)):
        rows = [x.clone(), f.clone()]
        block.join_forward(*rows, rows[first], rows[second], gate=gate, seed=1)
        assert torch.equal(rows[first], y) and torch.equal(rows[second], n)
    for to_x, to_f in ((0, 2), (1, 0), (1, 2), (0, 1)):
        rows = [dn.clone(), dr.clone(), f.clone()]
        block.join_backward(rows[0], rows[1], y, rows[2], rows[to_x], rows[to_f], gate=gate, seed=1)
        assert torch.equal(rows[to_x], dx) and torch.equal(rows[to_f], df)


@pytest.mark.parametrize("mode", MODES)
def test_join_rows_of_zeros(torch, L, mode):
    """A row of zeros has the norm zero, and its gradient is what eps leaves of it."""
    block = L.ccdc_block(64, 8, mode, eps=0.25).bind([5]).upload()
    z = torch.zeros(5, 64, dtype=block.dtype, device="cuda")
    y, n, dx, df = (torch.full_like(z, float("nan")) for _ in range(4))
    one = torch.ones_like(z)
    block.join_forward(z, z, y, n)
    block.join_backward(one, None, z, z, dx, df)
    torch.cuda.synchronize()
    assert (y == 0).all() and (n == 0).all() and (dx == 2).all() and (df == 4).all()


# ------------------------------------------------------------------ gradients against differences
def test_gradients_against_differences(torch, L):
    """The whole block, two joins around the feed-forward part, in fp32: the loss's change along a direction against the
    gradients' product with it, for every input and parameter.  Central differences with steps of 2^-6 of values around one:
    their own error is the third derivative times 2^-12 / 6, and the loss's 32-bit roundings over 2^-5; both are taken
    from the definition in 64 bits, whose difference quotient the gradients are held to, with 1e-4 of the terms' size for
    what 32 bits carry."""
    rng = np.random.default_rng(5)
    d, F, lengths, eps = 40, 56, [6, 0, 9], 1e-3
    N, M, mode = 3, 15, "f32"
    block = L.ccdc_block(d, F, mode, eps=eps, residual_scale=0.9, dropout_hidden=0.2, dropout_out=0.1).bind(lengths).upload()
    kh, ko = (R.factors(lengths, range(N), c, float(np.float32(p)), s, SEED) for c, p, s in ((F, 0.2, 0), (d, 0.1, 1)))
    names = ["x", "w_pre", "W_in", "W_out", "w_post", "gate", "w_next"]
    shapes = [(M, d), (d,), (2 * F, d), (d, F), (d,), (d,), (d,)]
    t, v = {}, {}
    for name, shape in zip(names, shapes):
        t[name], v[name] = numbers(torch, mode, rng, shape, 0.2 if len(shape) == 2 and name != "x" else 1.0)
    weight_n, weight_y = rng.normal(0, 1, (M, d)), rng.normal(0, 1, (M, d))

    def loss(**p):
        """Every parameter has a row a file."""
        per = lambda q: np.repeat(q, lengths, 0)  # noqa: E731
        hat, _ = R.normed(p["x"], eps32, False)
        n = hat * per(p["w_pre"])
        a = np.einsum("mk,mfk->mf", n, per(p["W_in"]))
        q, _ = R.activation("silu", a[:, :F])
        f = np.einsum("mf,mcf->mc", q * a[:, F:] * kh, per(p["W_out"]))
        fhat, _ = R.normed(f, eps32, False)
        y = rho32 * p["x"] + per(p["gate"]) * ko * (fhat * per(p["w_post"]))
        yhat, _ = R.normed(y, eps32, False)
        return (yhat * per(p["w_next"]) * weight_n).sum() + (y * weight_y).sum()

    eps32, rho32 = float(np.float32(eps)), float(np.float32(0.9))
    new = lambda: torch.empty(M, d, device="cuda")  # noqa: E731
    n, f, y, n2 = new(), new(), new(), new()
    saved = torch.empty(block.saved_bytes, dtype=torch.uint8, device="cuda")
    scaled = L.ccdc_block(d, F, mode, eps=eps).bind(lengths).upload()       # the join before: x's norm alone
    scaled.join_forward(t["x"], None, None, n, w_pre=t["w_pre"])
    block.ffn_forward(n, t["W_in"], t["W_out"], f, saved=saved, seed=SEED)
    after = dict(w_post=t["w_post"], gate=t["gate"], w_pre=t["w_next"], seed=SEED)
    block.join_forward(t["x"], f, y, n2, **after)
    g = {k: torch.empty((N,) + s, device="cuda") for k, s in zip(names[1:], shapes[1:])}
    dn, dr = (torch.from_numpy(w.astype(np.float32)).cuda() for w in (weight_n, weight_y))
    weight_n, weight_y = dn.double().cpu().numpy(), dr.double().cpu().numpy()
    dres, df, dnorm, dx = new(), new(), new(), new()
    block.join_backward(dn, dr, y, f, dres, df, dw_post=g["w_post"], dgate=g["gate"], dw_pre=g["w_next"], **after)
    rows = torch.empty(N, 3 * F * d, device="cuda")
    dW_in, dW_out = rows[:, :2 * F * d].unflatten(1, (2 * F, d)), rows[:, 2 * F * d:].unflatten(1, (d, F))
    block.ffn_backward(n, t["W_in"], t["W_out"], saved, df, dnorm, dW_in, dW_out)
    scaled.join_backward(dnorm, dres, t["x"], None, dx, None, w_pre=t["w_pre"], dw_pre=g["w_pre"])
    g["x"], g["W_in"], g["W_out"] = dx, dW_in, dW_out
    base = {k: q if k == "x" else np.broadcast_to(q, (N,) + q.shape).copy() for k, q in v.items()}
    for name in names:
        gradient = g[name].double().cpu().numpy()
        for trial in range(2):
            way = rng.normal(0, 1, base[name].shape)
            step = 2.0 ** -16
            q = [loss(**{**base, name: base[name] + s * step * way}) for s in (1, -1)]
            want, got = (q[0] - q[1]) / (2 * step), (gradient * way).sum()
            assert abs(got - want) <= 1e-4 * np.abs(gradient * way).sum(), (name, got, want)


# ------------------------------------------------------------------ dropout
@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("columns", [1, 7, 8, 100, 2049, 4160])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.9999, 1.0])
def test_dropout(torch, L, mode, columns, p):
    rng = np.random.default_rng(columns)
    lengths, ids = [3, 0, 14, 1], [9, 1, 0, (1 << 31) - 1]
    block = L.ccdc_block(8, 8, mode).bind(lengths, ids).upload()
    x, xv = numbers(torch, mode, rng, (18, columns), ld=columns + 3)
    res, rv = numbers(torch, mode, rng, (18, columns))
    keep = R.factors(lengths, ids, columns, p, 77, SEED).astype(np.float32)
    kept = xv.astype(np.float32) * keep
    for residual, want in ((None, kept), (res, kept + rv.astype(np.float32))):
        y = torch.full((18, columns), float("nan"), dtype=x.dtype, device="cuda")
        block.dropout(x, y, p, site=77, seed=SEED, residual=residual)
        # fp32 may multiply and add in one rounding: a unit in the last place of the sum's terms
        exact = torch.from_numpy(want).to(x.dtype).double().numpy()
        off = np.abs(y.double().cpu().numpy() - exact)
        slack = 0.0 if residual is None else 2 * R.ROUND[mode] * np.abs(exact) + 2.0 ** -23 * (np.abs(kept) + np.abs(rv))
        assert (off <= slack).all()
    block.dropout(x, x, p, site=77, seed=SEED)
    torch.cuda.synchronize()
    assert np.array_equal(x.double().cpu().numpy(), torch.from_numpy(kept).to(x.dtype).double().numpy())


def test_dropout_takes_out_what_is_no_number(torch, L):
    block = L.ccdc_block(8, 8, "f32").bind([64]).upload()
    x = torch.full((64, 512), float("inf"), device="cuda")
    x[:, ::2] = float("nan")
    y = torch.empty_like(x)
    block.dropout(x, y, 0.5, site=1, seed=3)
    gone = torch.from_numpy(R.factors([64], [0], 512, 0.5, 1, 3) == 0).cuda()
    assert (y[gone] == 0).all() and not torch.isfinite(y[~gone]).any()


# ------------------------------------------------------------------ streams, graphs, refusals
def test_calls_on_two_streams(torch, L):
    """The block's workspace is handed from stream to stream in the order of the calls."""
    rng = np.random.default_rng(2)
    block = L.ccdc_block(512, 1024, "bf16").bind([600]).upload()
    W_in, _ = numbers(torch, "bf16", rng, (2048, 512), 1 / 22)
    W_out, _ = numbers(torch, "bf16", rng, (512, 1024), 1 / 32)
    xs = [numbers(torch, "bf16", rng, (600, 512))[0] for _ in range(8)]
    alone = []
    for x in xs:
        y = torch.empty_like(x)
        block.ffn_forward(x, W_in, W_out, y)
        alone.append(y)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    ys = [torch.empty_like(x) for x in xs]
    torch.cuda.synchronize()
    for i, x in enumerate(xs):
        block.ffn_forward(x, W_in, W_out, ys[i], stream=streams[i % 2])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(alone, ys))


@pytest.mark.parametrize("mode", MODES)
def test_native_and_python_marshalling_agree(torch, L, mode):
    """A call on torch's current stream is handed over natively, one that names a stream through ctypes: the same arguments."""
    rng = np.random.default_rng(6)
    d, F, lengths = 72, 88, [5, 0, 20]
    block = L.ccdc_block(d, F, mode, dropout_hidden=0.1, dropout_out=0.2, residual_scale=0.5).bind(lengths).upload()
    x, dy = (numbers(torch, mode, rng, (25, d), ld=d + 8)[0] for _ in range(2))
    W_in, W_out = numbers(torch, mode, rng, (2 * F, d), 0.1)[0], numbers(torch, mode, rng, (d, F), 0.1)[0]
    w, gate = numbers(torch, mode, rng, (d,))[0], numbers(torch, mode, rng, (3, d))[0]
    saved = torch.empty(block.saved_bytes, dtype=torch.uint8, device="cuda")
    quick, taken = block._quick, []

    def watched(*args):
        taken.append(quick(*args))
        return taken[-1]

    block._quick = watched
    results = []
    for stream in (None, torch.cuda.current_stream()):
        y, z, n, dx, df, k = (empty(torch, x, 25, d, ld=d + 8) for _ in range(6))
        rows, sums = empty(torch, x, 3, 3 * F * d + 4), empty(torch, x, 3, 3 * d)
        dW_in, dW_out = rows[:, :2 * F * d].unflatten(1, (2 * F, d)), rows[:, 2 * F * d:3 * F * d].unflatten(1, (d, F))
        block.ffn_forward(x, W_in, W_out, y, saved=saved, seed=SEED, stream=stream)
        block.join_forward(x, y, z, n, w_post=w, gate=gate, w_pre=w, seed=SEED, stream=stream)
        block.join_backward(dy, None, z, y, dx, df, w_post=w, gate=gate, w_pre=w, dw_post=sums[:, :d], dgate=sums[:, d:2 * d],
                            dw_pre=sums[:, 2 * d:], seed=SEED, stream=stream)
        block.ffn_backward(x, W_in, W_out, saved, df, dx, dW_in, dW_out, stream=stream)
        block.dropout(x, k, 0.25, site=9, seed=SEED, residual=dy, stream=stream)
        torch.cuda.synchronize()
        results.append([t.clone() for t in (y, z, n, dx, df, k, rows[:, :3 * F * d], sums)])
    assert taken == [0] * 5
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_a_training_step_in_a_graph(torch, L):
    rng = np.random.default_rng(4)
    d, F, lengths, mode = 136, 256, [50, 0, 33], "bf16"
    block = L.ccdc_block(d, F, mode, dropout_hidden=0.1, dropout_out=0.1).bind(lengths).upload()
    x, dy = (numbers(torch, mode, rng, (83, d))[0] for _ in range(2))
    W_in, _ = numbers(torch, mode, rng, (2 * F, d), 1 / 12)
    W_out, _ = numbers(torch, mode, rng, (d, F), 1 / 16)
    saved = torch.empty(block.saved_bytes, dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(x) for _ in range(4)] + [torch.empty(3, 2 * F, d, dtype=x.dtype, device="cuda"),
                                                      torch.empty(3, d, F, dtype=x.dtype, device="cuda")]
    rows = torch.empty(3, 3 * F * d + 2 * d, dtype=x.dtype, device="cuda")
    dW_in, dW_out = rows[:, :2 * F * d].unflatten(1, (2 * F, d)), rows[:, 2 * F * d:3 * F * d].unflatten(1, (d, F))
    dgate, dw = rows[:, 3 * F * d:3 * F * d + d], rows[:, 3 * F * d + d:]

    def step():
        y, dx, z, n = outs[:4]
        block.ffn_forward(x, W_in, W_out, y, saved=saved, seed=7)
        block.join_forward(x, y, z, n, seed=7)
        block.join_backward(dy, dy, z, y, dx, n, dgate=dgate, dw_pre=dw, seed=7)
        block.ffn_backward(x, W_in, W_out, saved, n, dx, dW_in, dW_out)

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs[:4] + [rows]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        for t in outs[:4] + [rows]:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs[:4] + [rows]))
        x.mul_(1.0)                                  # the program's own work between replays
        torch.cuda.synchronize()


def test_refusals_of_calls(torch, L):
    B = L.binding
    d, F = 32, 48
    block = L.ccdc_block(d, F, "bf16").bind([4, 6]).upload()
    new = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    x, W_in, W_out, y = new(10, d), new(2 * F, d), new(d, F), new(10, d)
    saved = torch.zeros(block.saved_bytes, dtype=torch.uint8, device="cuda")
    for bad in ((new(10, d + 1), W_in, W_out, y), (x, new(F, d), W_out, y), (x, W_in, new(F, d), y), (x, W_in, W_out, new(9, d)),
                (x.float(), W_in, W_out, y), (x.cpu(), W_in, W_out, y), (new(d, 10).t(), W_in, W_out, y)):
        with pytest.raises(ValueError):
            block.ffn_forward(*bad)
    with pytest.raises(ValueError):
        block.ffn_forward(x, W_in, W_out, y, saved=saved[:-1])
    with pytest.raises(L.CcdcError) as e:
        block.ffn_forward(x[:9], W_in, W_out, y[:9], saved=saved)
    assert e.value.status == B.EINVAL
    with pytest.raises(L.CcdcError) as e:
        block.ffn_forward(new(11, d), W_in, W_out, new(11, d))
    assert e.value.status == B.EINVAL
    with pytest.raises(ValueError):
        block.ffn_backward(x, W_in, W_out, saved, y, None, new(3, 2 * F, d), new(2, d, F))        # a gradient a file
    with pytest.raises(L.CcdcError):
        block.ffn_backward(x, W_in, W_out, saved, y, None, new(2, 2 * F, d), None)                # one without the other
    with pytest.raises(L.CcdcError):
        block.ffn_backward(x, W_in, W_out, saved, y, None, None, None)                            # nothing wanted
    with pytest.raises(ValueError):
        block.join_forward(x, new(10, 2 * d)[:, :d], y, None)                                     # another stride
    with pytest.raises(L.CcdcError):
        block.join_forward(x, None, None, None)
    with pytest.raises(L.CcdcError):
        block.join_backward(None, None, y, x, x, x)
    with pytest.raises(L.CcdcError):
        block.join_backward(x, None, None, None, x, None)
    for p in (-0.1, 1.5, float("nan")):
        with pytest.raises(L.CcdcError):
            block.dropout(x, y, p, site=0)
    lib, ptr = L.load_library(), lambda t: t.data_ptr()
    st = torch.cuda.current_stream().cuda_stream
    call = lambda **k: lib.ccdc_ffn_forward(*{"b": block._h, "rows": 10, "x": ptr(x), "ldx": d, "wi": ptr(W_in), "wo": ptr(W_out),  # noqa: E731
                                              "y": ptr(y), "ldy": d, "s": None, "seed": 0, "st": st, **k}.values())
    assert call() == B.OK
    for k in ({"x": None}, {"x": ptr(x) + 1}, {"ldx": d - 1}, {"ldy": 0}, {"rows": -1}, {"y": None}, {"wi": None}, {"b": None},
              {"s": ptr(saved) + 8}):
        assert call(**k) == B.EINVAL, k
    wide = L.ccdc_block(20000, 8, "bf16").bind([1]).upload()
    w = new(1, 20000)
    with pytest.raises(L.CcdcError) as e:
        wide.join_forward(w, None, None, w)
    assert e.value.status == B.ESIZE
    torch.cuda.synchronize()
