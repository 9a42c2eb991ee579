"""The trained block in 64 bits, from its definitions (include/ccdc.h), with a bound on how far a correct implementation may
be from each result.  Test infrastructure only; shares no code with the library.

Bounds are worst cases, element by element, of these roundings and no others:
  u    one rounding to the element type: of every result, of h and of the gradients of a and u where they are stored
       between two products (16-bit types), relative, plus half the smallest subnormal
  e    everything carried in 32 bits: a sum of K terms is at most K 2^-24 of the sum of their magnitudes off, in any order;
       e = (K + 64) 2^-23 is twice that, with room for the few operations before and after (an activation, a product of
       three parts) at 2^-24 each
An error made earlier is carried through the formula that uses the value."""
import numpy as np
from scipy.special import erf, expit

ROUND = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}      # bf16 has 8 bits of significand, f16 11
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25}


def philox(counter, key):
    """Philox4x32-10 on arrays of 32-bit numbers: [..., 4], (low, high) -> [..., 4]."""
    c = [np.asarray(counter[..., i], dtype=np.uint64) for i in range(4)]
    k0, k1 = int(key[0]), int(key[1])
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, -1).astype(np.uint32)


def factors(lengths, ids, columns, p, site, seed):
    """Dropout's factor of every element of the batch, [M][columns]."""
    thr = int(np.floor(np.float64(p) * 65536 + 0.5))
    token = np.concatenate([np.arange(n) for n in lengths] + [np.zeros(0, int)])
    number = np.repeat(np.asarray(ids), lengths)
    counter = np.zeros((len(token), columns, 4), np.uint64)
    counter[..., 0] = np.arange(columns)[None, :] // 8
    counter[..., 1], counter[..., 2], counter[..., 3] = token[:, None], number[:, None], site
    words = philox(counter, (seed & 0xFFFFFFFF, seed >> 32))
    c = np.arange(columns)
    word = np.take_along_axis(words, np.broadcast_to((c % 8 // 2)[None, :, None], (len(token), columns, 1)), -1)[..., 0]
    half = (word >> (16 * (c % 2))[None, :].astype(np.uint32)) & np.uint32(0xFFFF)
    return np.where(half >= thr, 65536.0 / (65536 - thr) if thr < 65536 else 0.0, 0.0)


def activation(name, a):
    """The activation, its derivative, and bounds on the slopes of both."""
    if name == "silu":
        s = expit(a)
        return a * s, s + a * s * (1 - s)
    if name == "gelu":
        cdf = 0.5 * (1 + erf(a / np.sqrt(2)))
        return a * cdf, cdf + a * np.exp(-a * a / 2) / np.sqrt(2 * np.pi)
    return np.maximum(a, 0), (a > 0).astype(float)


def spans(lengths):
    ends = np.cumsum(lengths)
    return [slice(e - n, e) for e, n in zip(ends, lengths)]


def ffn(lengths, x, W_in, W_out, dy, keep, act, mode):
    """{name: (value, bound)} of y, h and, with dy, of dx, dW_in, dW_out."""
    u, tiny = ROUND[mode], TINY[mode]
    F, d = W_in.shape[0] // 2, x.shape[1]
    A = np.abs
    e = lambda K: (K + 64) * 2.0 ** -23  # noqa: E731
    inner = u if mode != "f32" else 0.0                     # h and the gradients of a and u are stored
    au, Bau = x @ W_in.T, e(d) * (A(x) @ A(W_in).T)
    a, v, Ba, Bv = au[:, :F], au[:, F:], Bau[:, :F], Bau[:, F:]
    q, slope = activation(act, a)
    # |activation'| < 1.2 and |activation''| < 1 for all three (relu's slope jumps at 0)
    Bq, Bs = 1.2 * Ba + e(0) * A(q), 1.0 * Ba + e(0) * A(slope) + ((act == "relu") & (A(a) <= Ba))
    h = q * v * keep
    Bh = keep * (Bq * A(v) + A(q) * Bv + Bq * Bv) + (e(0) + inner) * A(h) + tiny
    y = h @ W_out.T
    out = {"h": (h, Bh), "y": (y, Bh @ A(W_out).T + e(F) * (A(h) @ A(W_out).T) + u * A(y) + tiny)}
    if dy is None:
        return out
    dh, Bdh = dy @ W_out, e(d) * (A(dy) @ A(W_out))
    P, BP = slope * v * keep, keep * (Bs * A(v) + A(slope) * Bv + Bs * Bv)
    Q, BQ = q * keep, keep * Bq
    dau = np.concatenate((dh * P, dh * Q), 1)
    Bdau = np.concatenate((Bdh * (A(P) + BP) + A(dh) * BP, Bdh * (A(Q) + BQ) + A(dh) * BQ), 1) + (e(0) + inner) * A(dau) + tiny
    dx = dau @ W_in
    out["dx"] = dx, Bdau @ A(W_in) + e(2 * F) * (A(dau) @ A(W_in)) + u * A(dx) + tiny
    W1, B1, W2, B2 = [], [], [], []
    for s in spans(lengths):
        n = s.stop - s.start
        W1.append(dau[s].T @ x[s])
        B1.append(Bdau[s].T @ A(x[s]) + e(n) * (A(dau[s]).T @ A(x[s])) + u * A(W1[-1]) + tiny)
        W2.append(dy[s].T @ h[s])
        B2.append(A(dy[s]).T @ Bh[s] + e(n) * (A(dy[s]).T @ A(h[s])) + u * A(W2[-1]) + tiny)
    out["dW_in"], out["dW_out"] = (np.stack(W1), np.stack(B1)), (np.stack(W2), np.stack(B2))
    return out


def normed(v, eps, centred):
    if centred:
        v = v - v.mean(1, keepdims=True)
    rstd = 1 / np.sqrt((v * v).mean(1, keepdims=True) + eps)
    return v * rstd, rstd


def norm_gradient(e, hat, rstd, centred):
    g = e - hat * (e * hat).mean(1, keepdims=True)
    size = np.abs(e) + np.abs(hat) * np.abs(e * hat).mean(1, keepdims=True)
    if centred:
        g, size = g - e.mean(1, keepdims=True), size + np.abs(e).mean(1, keepdims=True)
    return rstd * g, rstd * size


def join(x, f, w_post, gate, w_pre, keep, rho, eps, centred, mode):
    """{name: (value, bound)} of y and n.  A norm's value is at most e of the largest of its row's values off, relative to its
    own size where nothing is subtracted: bounds take 4 e of the row's scale."""
    u, tiny, d = ROUND[mode], TINY[mode], x.shape[1]
    e = (d + 64) * 2.0 ** -23
    y, size = rho * x, np.abs(rho * x)
    if f is not None:
        hat, rstd = normed(f, eps, centred)
        scale = (np.abs(f) + (np.abs(f).mean(1, keepdims=True) if centred else 0)) * rstd
        y = y + gate * keep * (hat * w_post)
        size = size + np.abs(gate * keep * w_post) * scale
    B = 4 * e * size
    out = {"y": (y, B + u * np.abs(y) + tiny)}
    hat, rstd = normed(y, eps, centred)
    # n follows y by at most rstd, its row's mean and norm by the mean of y's errors
    Bn = np.abs(w_pre) * rstd * (B + B.mean(1, keepdims=True) + np.abs(hat) * np.sqrt((B * B).mean(1, keepdims=True)))
    Bn += 4 * e * np.abs(w_pre) * rstd * (np.abs(y) + (np.abs(y).mean(1, keepdims=True) if centred else 0))
    n = hat * w_pre
    out["n"] = n, Bn + u * np.abs(n) + tiny
    return out


def join_gradient(lengths, dn, dr, y, f, w_post, gate, w_pre, keep, rho, eps, centred, mode):
    """{name: (value, bound)} of dx, df and the per-file gradients, at y as it is stored."""
    u, tiny = ROUND[mode], TINY[mode]
    d = (y if y is not None else dr).shape[1]
    e = (d + 64) * 2.0 ** -23
    A, out = np.abs, {}
    dy = np.zeros((sum(lengths), d)) if dr is None else dr
    B = e * A(dy)
    sums = lambda t: np.stack([t[s].sum(0) for s in spans(lengths)])  # noqa: E731

    def learned(name, value, size):
        """Sums over a file's rows: every term at most 8 e of its size off, the sum as any in 32 bits."""
        total, magnitude = sums(value), sums(size)
        more = np.asarray([(n + 64) * 2.0 ** -23 for n in lengths])[:, None]
        out[name] = total, (8 * e + more) * magnitude + u * A(total) + tiny

    if dn is not None:
        hat, rstd = normed(y, eps, centred)
        scale = (A(y) + (A(y).mean(1, keepdims=True) if centred else 0)) * rstd
        g, size = norm_gradient(dn * w_pre, hat, rstd, centred)
        _, wide = norm_gradient(A(dn * w_pre), scale, rstd, True)
        dy, B = dy + g, B + 8 * e * np.maximum(size, wide)
        learned("dw_pre", dn * hat, A(dn) * scale)
    out["dx"] = rho * dy, A(rho) * B + u * A(rho * dy) + e * A(rho * dy) + tiny
    if f is None:
        return out
    hat, rstd = normed(f, eps, centred)
    scale = (A(f) + (A(f).mean(1, keepdims=True) if centred else 0)) * rstd
    kd, Bk = keep * dy, keep * B
    g, size = norm_gradient(kd * gate * w_post, hat, rstd, centred)
    _, wide = norm_gradient((A(kd) + Bk) * A(gate * w_post), scale, rstd, True)
    _, carried = norm_gradient(Bk * A(gate * w_post), scale, rstd, True)
    out["df"] = g, 8 * e * np.maximum(size, wide) + carried + u * A(g) + tiny
    learned("dw_post", kd * gate * hat, (A(kd) + Bk / (8 * e)) * A(gate) * scale)
    learned("dgate", kd * w_post * hat, (A(kd) + Bk / (8 * e)) * A(w_post) * scale)
    return out
