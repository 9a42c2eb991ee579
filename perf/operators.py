"""The operators of a trained block whose per-file gradients feed the shuffle, as measurable cases: a gated feed-forward
block, the join of one block with the next (norm, gate, dropout, residual, next norm) and dropout from a counter-based
generator, with their gradients.

A batch is M tokens of N files, one file after the other; the gradients of what is learned are one row per file (the
values V that the shuffle path codes and sums).  With d the width, F the hidden size, file n(m) and token t(m) of row m:

  ffn      a = x Wg', u = x Wu', h = D(act(a) u), y = h Wd';  W_in = [Wg; Wu] is [2F][d], W_out = Wd is [d][F]
  join     y = rho x + gate D(norm(f; w_post)),  n = norm(y; w_pre)
  dropout  y = D(x)

D keeps element (m, c) where halfword c % 8 of Philox4x32-10 on the counter (c / 8, t(m), n(m), site) and the key (seed)
is at least thr = rint(65536 p), times 65536 / (65536 - thr).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False             # True: the package's operators; False: the plain form

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6
LAYER = 3               # the block's number: dropout of the hidden values is site 2 LAYER, of the join 2 LAYER + 1
SITE = 11               # site of the dropout called by itself


# ------------------------------------------------------------------ cases
def _ffn(what, files, tokens, width, hidden, mode, act="silu", p=0.0, ragged=False):
    return {"op": "ffn", "what": what, "files": files, "tokens": tokens, "ragged": ragged, "width": width,
            "hidden": hidden, "mode": mode, "act": act, "p": p}


def _join(what, files, tokens, width, mode, p=0.0, ragged=False, centred=False, gate="shared"):
    return {"op": "join", "what": what, "files": files, "tokens": tokens, "ragged": ragged, "width": width,
            "mode": mode, "p": p, "centred": centred, "gate": gate}


def _dropout(files, tokens, width, mode, p, ragged=False):
    return {"op": "dropout", "what": "forward", "files": files, "tokens": tokens, "ragged": ragged, "width": width,
            "mode": mode, "p": p}


def listed():
    """`tokens` are those of a file, on average where the files are ragged."""
    return [
        # answering one token: the weights of a 25.6M-parameter block are read once, latency counts
        {"name": "ffn_one_token_bf16", **_ffn("forward", 1, 1, 2048, 4160, "bf16")},
        # a few requests at once
        {"name": "ffn_batch_f16", **_ffn("forward", 24, 1, 1600, 4400, "f16", "gelu")},
        # a long prompt through a large block: the largest forward
        {"name": "ffn_prompt_bf16", **_ffn("forward", 1, 8192, 4096, 11264, "bf16")},
        # a training step: 28 files (one per pair of 8 nodes) mapped to 28 gradients of 25.6M parameters, 1.4 GB of V
        {"name": "ffn_train_bf16", **_ffn("train", 28, 512, 2048, 4160, "bf16", p=0.1)},
        # the same in 32 bits on fewer, uneven files and a smaller block
        {"name": "ffn_train_f32", **_ffn("train", 10, 300, 1024, 2600, "f32", "gelu", ragged=True)},
        # sizes that divide by nothing, many short uneven files, some of them empty
        {"name": "ffn_train_ragged_bf16", **_ffn("train", 56, 37, 515, 1333, "bf16", p=0.2, ragged=True)},
        # between two blocks while answering: a handful of rows, latency
        {"name": "join_tokens_bf16", **_join("forward", 8, 1, 2048, "bf16")},
        # between two blocks of a long prompt
        {"name": "join_prompt_f16", **_join("forward", 1, 16384, 4096, "f16")},
        # training, forward and backward with dropout, per-file gradients of both norms and the gate
        {"name": "join_train_bf16", **_join("train", 28, 512, 2048, "bf16", 0.1)},
        {"name": "join_train_ragged_f32", **_join("train", 45, 300, 1001, "f32", 0.1, True, True, "files")},
        # dropout by itself: of the embedded tokens of a step, and of a large hidden state
        {"name": "dropout_tokens_f32", **_dropout(20, 33, 1000, "f32", 0.1, True)},
        {"name": "dropout_hidden_bf16", **_dropout(28, 512, 4160, "bf16", 0.1)},
    ]


def draw(rng):
    """One more case of the same ranges: one token to 16384, widths of 64 to 4096 (dropout, join: 8192), whole packs or
    odd, one to 64 files, equal or uneven.  None costs more than the largest listed one."""
    top = {"flops": 18 * 28 * 512 * 2048 * 4160, "bytes": 1.7e9}

    def size(low, high, grain):
        """An odd multiple of the grain: how far a size divides is what the grain says."""
        v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
        return ((v // grain - 1) | 1) * grain if v >= grain else v

    while True:
        op = rng.choices(["ffn", "join", "dropout"], [5, 3, 1])[0]
        mode = rng.choice(["bf16", "bf16", "f16", "f32"])
        grain, some = rng.choice([512, 64, 64, 8, 1]), rng.choice([1, 1, 16])
        what = rng.choice(["forward", "train"])
        files, ragged = size(1, 64, 1), rng.random() < 0.5
        p = rng.choice([0.0, 0.1, 0.3])
        if op == "ffn" and what == "forward":
            few = rng.random() < 0.5                       # half of them answer a few tokens
            files, tokens = (size(1, 64, 1), 1) if few else (1, size(1, 8192, some))
            width = size(256, 4096, grain)
            case = _ffn(what, files, tokens, width, size(2 * width, 3 * width, grain), mode,
                        rng.choice(["silu", "gelu", "relu"]))
        elif op == "ffn":
            width = size(128, 2048, grain)
            case = _ffn(what, files, size(8, 2048, some), width, size(1.5 * width, 4 * width, grain), mode,
                        rng.choice(["silu", "gelu", "relu"]), p, ragged)
        elif op == "join":
            case = _join(what, files, size(1, 4096, some), size(64, 8192, grain), mode, p, ragged, rng.random() < 0.3,
                         rng.choice(["shared", "files", "none"]))
        else:
            case = _dropout(files, size(1, 4096, some), size(64, 8192, grain), mode, rng.choice([0.1, 0.3, 0.5]), ragged)
        need = work(case)
        kept = _tokens(case) * case.get("hidden", case["width"])
        if need["flops"] <= top["flops"] and need["bytes"] <= top["bytes"] and kept <= 8192 * 11264:
            return case


def _lengths(case):
    """Tokens of each file.  Uneven files: from none to about twice the average, by a fixed pattern; the last takes the rest."""
    n, each = case["files"], case["tokens"]
    if not case["ragged"] or n == 1:
        return [each] * n
    got = [each * (7 * i * i + 3 * i) % (2 * each + 1) for i in range(n - 1)]
    return got + [max(0, n * each - sum(got))]


def _tokens(case):
    return sum(_lengths(case))


def work(case):
    M, N, d, eb = _tokens(case), case["files"], case["width"], BYTES[case["mode"]]
    if case["op"] == "ffn":
        F = case["hidden"]
        if case["what"] == "forward":
            return {"bytes": (2 * M * d + 3 * d * F) * eb, "flops": 6 * M * d * F}
        # x, y, dy, dx; the weights; their gradients for every file
        return {"bytes": (4 * M * d + 3 * d * F + 3 * N * d * F) * eb, "flops": 18 * M * d * F}
    if case["op"] == "join":
        gates = {"none": 0, "shared": 1, "files": N}[case["gate"]]
        if case["what"] == "forward":
            return {"bytes": (4 * M * d + (2 + gates) * d) * eb, "flops": 12 * M * d}
        learned = 2 + (case["gate"] != "none")
        # x and f read once, y and n written; then dn and dr read, dx and df written
        return {"bytes": (8 * M * d + (2 + gates + learned * N) * d) * eb, "flops": 40 * M * d}
    return {"bytes": 2 * M * d * eb, "flops": M * d}


# ------------------------------------------------------------------ inputs
def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype, M, d, N = TYPES[case["mode"]], _tokens(case), case["width"], case["files"]

    def normal(*shape, std=1.0, mean=0.0):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, std, generator=g).to(dtype)

    s = {"key": int(seed) * 0x9E3779B97F4A7C15 % (1 << 64)}
    if case["op"] == "dropout":
        s["x"] = normal(M, d)
        return s
    if case["op"] == "ffn":
        F = case["hidden"]
        s["x"] = normal(M, d)                             # what a norm gives
        s["W_in"] = normal(2 * F, d, std=1 / math.sqrt(d))
        s["W_out"] = normal(d, F, std=1 / math.sqrt(F))
        if case["what"] == "train":
            s["dy"] = normal(M, d, std=0.05)
        return s
    # a residual stream has a few channels that are much larger than the others
    loud = 1 + 7 * (torch.rand(d, device="cuda", generator=g) < 0.02).float()
    s["x"] = (normal(M, d, std=1.5).float() * loud).to(dtype)
    s["f"] = normal(M, d, std=0.7, mean=0.05)
    s["w_post"], s["w_pre"] = normal(d, std=0.2, mean=1.0), normal(d, std=0.2, mean=1.0)
    s["gate"] = {"none": lambda: None, "shared": lambda: normal(d, std=0.3, mean=0.5),
                 "files": lambda: normal(N, d, std=0.3, mean=0.5)}[case["gate"]]()
    if case["what"] == "train":
        s["dn"], s["dr"] = normal(M, d, std=0.05), normal(M, d, std=0.02)
    return s


RHO = 0.8               # the residual scale


def prepare(case, seed):
    """The inputs, the parameters, the buffers that a program keeps for results, and the rows' files: as tables on the
    device, and in the package's handle where that is what runs."""
    s = {"case": case, **_inputs(case, seed)}
    dtype, M, d, N, lengths = TYPES[case["mode"]], _tokens(case), case["width"], case["files"], _lengths(case)
    new = lambda *shape: torch.zeros(shape, dtype=dtype, device="cuda")  # noqa: E731
    s["y"] = new(M, d)
    if case["op"] == "join":
        s["n"] = new(M, d)
    if case["what"] == "train":
        if case["op"] == "ffn":
            F = case["hidden"]
            s["dx"], s["V"] = new(M, d), new(N, 3 * F * d)             # a file's row: dW_in, then dW_out
            s["dW_in"], s["dW_out"] = s["V"][:, :2 * F * d].view(N, 2 * F, d), s["V"][:, 2 * F * d:].view(N, d, F)
        else:
            s["dx"], s["df"], s["V"] = new(M, d), new(M, d), new(N, 3 * d)
            s["dw_pre"], s["dw_post"], s["dgate"] = s["V"][:, :d], s["V"][:, d:2 * d], s["V"][:, 2 * d:]
    at = torch.tensor(lengths, device="cuda")
    s["file"] = torch.repeat_interleave(torch.arange(N, device="cuda"), at, output_size=M)       # of each row
    s["token"] = torch.arange(M, device="cuda") - (at.cumsum(0) - at)[s["file"]]
    s["longest"] = max(lengths)
    s["block"] = _handle(case, lengths) if own else None
    if own and case["what"] == "train" and case["op"] == "ffn":
        s["saved"] = torch.empty(s["block"].saved_bytes, dtype=torch.uint8, device="cuda")
    return s


def _handle(case, lengths):
    import paper_1805_01993_amd as L
    block = L.ccdc_block(case["width"], case.get("hidden", 1), case["mode"], activation=case.get("act", "silu"),
                         norm="centred" if case.get("centred") else "rms", eps=EPS, residual_scale=RHO, layer=LAYER,
                         dropout_hidden=case["p"] if case["op"] == "ffn" else 0.0,
                         dropout_out=case["p"] if case["op"] == "join" else 0.0)
    return block.bind(lengths).upload()


# ------------------------------------------------------------------ one pass
def run(state):
    if own:
        return _run_own(state)
    return {"ffn": _plain_ffn, "join": _plain_join, "dropout": _plain_dropout}[state["case"]["op"]](state)


def _run_own(s):
    case, block = s["case"], s["block"]
    train = case["what"] == "train"
    if case["op"] == "dropout":
        block.dropout(s["x"], s["y"], case["p"], site=SITE, seed=s["key"])
        return {"y": s["y"]}
    if case["op"] == "ffn":
        block.ffn_forward(s["x"], s["W_in"], s["W_out"], s["y"], saved=s["saved"] if train else None, seed=s["key"])
        if not train:
            return {"y": s["y"]}
        block.ffn_backward(s["x"], s["W_in"], s["W_out"], s["saved"], s["dy"], s["dx"], s["dW_in"], s["dW_out"])
        return {k: s[k] for k in ("y", "dx", "dW_in", "dW_out")}
    learned = {"w_post": s["w_post"], "gate": s["gate"], "w_pre": s["w_pre"], "seed": s["key"]}
    block.join_forward(s["x"], s["f"], s["y"], s["n"], **learned)
    if not train:
        return {"y": s["y"], "n": s["n"]}
    gated = s["gate"] is not None
    block.join_backward(s["dn"], s["dr"], s["y"], s["f"], s["dx"], s["df"], dw_pre=s["dw_pre"], dw_post=s["dw_post"],
                        dgate=s["dgate"] if gated else None, **learned)
    return {k: s[k] for k in ("y", "n", "dx", "df", "dw_pre", "dw_post") + (("dgate",) if gated else ())}


# ------------------------------------------------------------------ the plain form: elementary operations in 32 bits
def _philox(c0, c1, c2, c3, key):
    """Philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011) on 32-bit numbers held in 64; products wrap, their bits are right."""
    k0, k1, low = key & 0xFFFFFFFF, key >> 32, 0xFFFFFFFF
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & low) ^ c1 ^ k0, p1 & low, ((p0 >> 32) & low) ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _kept(s, columns, p, site):
    """[M][columns]: the factor of every value, 0 or 1 / (1 - p)."""
    thr = int(round(p * 65536))
    if thr == 0:
        return 1.0
    unit = torch.arange(-(-columns // 8), device="cuda")[None, :]
    token, file = s["token"][:, None], s["file"][:, None]
    words = torch.stack(torch.broadcast_tensors(*_philox(unit, token, file, torch.full_like(unit, site), s["key"])), -1)
    halves = torch.stack((words & 0xFFFF, words >> 16), -1).reshape(token.shape[0], -1)[:, :columns]
    return (halves >= thr).float() * (65536 / (65536 - thr) if thr < 65536 else 0.0)


def _plain_dropout(s):
    x = s["x"].float()
    return {"y": (x * _kept(s, x.shape[1], s["case"]["p"], SITE)).to(s["x"].dtype)}


def _act(name, a):
    """The activation and its derivative."""
    if name == "silu":
        e = 1 / (1 + torch.exp(-a))
        return a * e, e * (1 + a * (1 - e))
    if name == "gelu":
        cdf = 0.5 * (1 + torch.erf(a * math.sqrt(0.5)))
        return a * cdf, cdf + a * torch.exp(-0.5 * a * a) * (1 / math.sqrt(2 * math.pi))
    return torch.clamp(a, min=0), (a > 0).float()


def _by_file(s, t):
    """[N][longest][columns]: the rows of each file, the rest zero."""
    out = torch.zeros(s["case"]["files"], max(1, s["longest"]), t.shape[1], device=t.device)
    out[s["file"], s["token"]] = t
    return out


def _plain_ffn(s):
    case, dtype, F = s["case"], s["x"].dtype, s["case"]["hidden"]
    x, W_in, W_out = s["x"].float(), s["W_in"].float(), s["W_out"].float()
    au = x @ W_in.t()
    a, u = au[:, :F], au[:, F:]
    act, slope = _act(case["act"], a)
    keep = _kept(s, F, case["p"], 2 * LAYER)
    h = act * u * keep
    y = h @ W_out.t()
    if case["what"] == "forward":
        return {"y": y.to(dtype)}
    dy = s["dy"].float()
    dh = (dy @ W_out) * keep
    dau = torch.cat((dh * u * slope, dh * act), 1)
    dx = dau @ W_in
    dW_in = torch.bmm(_by_file(s, dau).transpose(1, 2).contiguous(), _by_file(s, x))
    dW_out = torch.bmm(_by_file(s, dy).transpose(1, 2).contiguous(), _by_file(s, h))
    return {k: v.to(dtype) for k, v in (("y", y), ("dx", dx), ("dW_in", dW_in), ("dW_out", dW_out))}


def _normed(v, centred):
    """v hat, and the factor that made it."""
    if centred:
        v = v - v.mean(1, keepdim=True)
    rstd = torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)
    return v * rstd, rstd


def _norm_back(e, hat, rstd, centred):
    e_less = e - hat * (e * hat).mean(1, keepdim=True)
    return rstd * (e_less - e.mean(1, keepdim=True) if centred else e_less)


def _plain_join(s):
    case, dtype, centred = s["case"], s["x"].dtype, s["case"]["centred"]
    x, f, w_post, w_pre = (s[k].float() for k in ("x", "f", "w_post", "w_pre"))
    gate = 1.0 if s["gate"] is None else s["gate"].float()[s["file"]] if case["gate"] == "files" else s["gate"].float()
    keep = _kept(s, x.shape[1], case["p"], 2 * LAYER + 1)
    fhat, frstd = _normed(f, centred)
    z = fhat * w_post * keep
    y = RHO * x + gate * z
    yhat, _ = _normed(y, centred)
    out = {"y": y.to(dtype), "n": (yhat * w_pre).to(dtype)}
    if case["what"] == "forward":
        return out
    dn, dr = s["dn"].float(), s["dr"].float()
    yhat, yrstd = _normed(out["y"].float(), centred)       # a program has y as it was stored
    dy = dr + _norm_back(dn * w_pre, yhat, yrstd, centred)
    dz = gate * dy * keep
    df = _norm_back(dz * w_post, fhat, frstd, centred)
    per_file = lambda t: torch.zeros(case["files"], t.shape[1], device=t.device).index_add_(0, s["file"], t)  # noqa: E731
    out |= {"dx": RHO * dy, "df": df, "dw_pre": per_file(dn * yhat), "dw_post": per_file(dz * fhat)}
    if s["gate"] is not None:
        out["dgate"] = per_file(dy * z)
    return {k: v.to(dtype) for k, v in out.items()}


# ------------------------------------------------------------------ the same from the definitions, in 64 bits
def _factors(lengths, columns, p, site, key):
    """Dropout's factors [M][columns] by unsigned arithmetic on the host."""
    thr = int(np.rint(65536.0 * p))
    if thr == 0:
        return None
    u32, u64 = np.uint32, np.uint64
    units = (columns + 7) // 8
    shape = (sum(lengths), units)
    ctr = [np.broadcast_to(v, shape).astype(u32) for v in (
        np.arange(units)[None, :],
        np.concatenate([np.arange(n) for n in lengths])[:, None] if shape[0] else np.zeros((0, 1)),
        np.repeat(np.arange(len(lengths)), lengths)[:, None], np.full((1, 1), site))]
    k = [key & 0xFFFFFFFF, key >> 32]
    for _ in range(10):
        left, right = ctr[0].astype(u64) * u64(0xD2511F53), ctr[2].astype(u64) * u64(0xCD9E8D57)
        high = lambda v: (v >> u64(32)).astype(u32)  # noqa: E731
        ctr = [high(right) ^ ctr[1] ^ u32(k[0]), right.astype(u32), high(left) ^ ctr[3] ^ u32(k[1]), left.astype(u32)]
        k = [(k[0] + 0x9E3779B9) % (1 << 32), (k[1] + 0xBB67AE85) % (1 << 32)]
    halves = np.ascontiguousarray(np.stack(ctr, -1)).view(np.uint16).reshape(shape[0], units * 8)[:, :columns]
    keep = torch.from_numpy((halves >= thr).astype(np.uint8)).cuda().double()
    return keep * (65536.0 / (65536 - thr)) if thr < 65536 else keep * 0


def _sums_by_file(lengths, left, right):
    """left[n]' right[n] for every file's rows."""
    out = torch.zeros(len(lengths), left.shape[1], right.shape[1], dtype=torch.float64, device=left.device)
    at = 0
    for n, rows in enumerate(lengths):
        if rows:
            out[n] = left[at:at + rows].t().contiguous() @ right[at:at + rows]
        at += rows
    return out


def exact(case, seed):
    s, lengths, d = _inputs(case, seed), _lengths(case), case["width"]
    v = {k: t.double() for k, t in s.items() if isinstance(t, torch.Tensor)}
    if case["op"] == "dropout":
        keep = _factors(lengths, d, case["p"], SITE, s["key"])
        return {"y": v["x"] if keep is None else v["x"] * keep}
    if case["op"] == "ffn":
        F, name = case["hidden"], case["act"]
        keep = _factors(lengths, F, case["p"], 2 * LAYER, s["key"])
        a, u = v["x"] @ v["W_in"][:F].t().contiguous(), v["x"] @ v["W_in"][F:].t().contiguous()
        if name == "silu":
            act, slope = a * torch.sigmoid(a), torch.sigmoid(a) + a * torch.sigmoid(a) * torch.sigmoid(-a)
        elif name == "gelu":
            act = a * torch.special.ndtr(a)
            slope = torch.special.ndtr(a) + a * torch.exp(-a.square() / 2) / math.sqrt(2 * math.pi)
        else:
            act, slope = torch.where(a > 0, a, 0.0), torch.where(a > 0, 1.0, 0.0).double()
        if keep is not None:
            act, slope = act * keep, slope * keep
        h = act * u
        out = {"y": h @ v["W_out"].t().contiguous()}
        if case["what"] == "forward":
            return out
        dh = v["dy"] @ v["W_out"]
        da, du = dh * u * slope, dh * act
        out["dx"] = da @ v["W_in"][:F] + du @ v["W_in"][F:]
        out["dW_in"] = torch.cat((_sums_by_file(lengths, da, v["x"]), _sums_by_file(lengths, du, v["x"])), 1)
        out["dW_out"] = _sums_by_file(lengths, v["dy"], h)
        return out

    rows = torch.tensor(lengths, device="cuda")
    gate = torch.ones(d, dtype=torch.float64, device="cuda") if s["gate"] is None else v["gate"]
    if case["gate"] == "files":
        gate = torch.repeat_interleave(gate, rows, 0)
    keep = _factors(lengths, d, case["p"], 2 * LAYER + 1, s["key"])
    keep = 1.0 if keep is None else keep

    def norm(t, w):
        if case["centred"]:
            t = t - t.sum(1, keepdim=True) / d
        return t / torch.sqrt(t.square().sum(1, keepdim=True) / d + EPS) * w

    y = RHO * v["x"] + gate * keep * norm(v["f"], v["w_post"])
    out = {"y": y, "n": norm(y, v["w_pre"])}
    if case["what"] == "forward":
        return out
    # the gradients by differentiating the definition, at y as it is stored for each step
    stored = y.to(TYPES[case["mode"]]).double().requires_grad_()
    per_row = {k: v[k].expand(len(y), d).clone().requires_grad_() for k in ("w_pre", "w_post")}
    (dy,) = torch.autograd.grad(norm(stored, v["w_pre"]), stored, v["dn"])
    dy = dy + v["dr"]
    (dw_pre,) = torch.autograd.grad(norm(stored.detach(), per_row["w_pre"]), per_row["w_pre"], v["dn"])
    f, gates = v["f"].requires_grad_(), gate.expand(len(y), d).clone().requires_grad_()
    df, dw_post, dgate = torch.autograd.grad(gates * keep * norm(f, per_row["w_post"]), (f, per_row["w_post"], gates), dy)
    ones = torch.ones(len(y), 1, dtype=torch.float64, device="cuda")
    per_file = lambda t: _sums_by_file(lengths, ones, t)[:, 0]  # noqa: E731
    out |= {"dx": RHO * dy, "df": df, "dw_pre": per_file(dw_pre), "dw_post": per_file(dw_post)}
    if s["gate"] is not None:
        out["dgate"] = per_file(dgate)
    return out
