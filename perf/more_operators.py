"""Learning from a teacher that answers in 8 bits, as measurable cases: matrices held in 8-bit floating point with a scale for
each block of 128, their product, the top logits of what the teacher answers, and the distillation of a student from them with
its gradient.

  quantise  of each row, blocks of 128 columns: e the least whole number with max |x| <= 448 2^e (0 where the block is zero,
            at least -127), q = x 2^-e rounded to e4m3; rows are padded with zeros to whole blocks.  The scale is kept as e + 127,
            a row's blocks padded to a multiple of four with 127.
  product   y[m][n] = sum over blocks b of 2^(ex[m][b] + ew[n][b]) sum over the block's k of qx[m][k] qw[n][k]
  top       of each row, the k largest logits and their columns, larger ones first and of equal ones the lower column (-1 and
            -inf where a row has fewer above -inf), and rest = log of the sum of exp(z / T) over the columns not among them
  distill   p = softmax of (t_1 / T ... t_k / T, rest) (no last one where rest is not given), q = softmax(z / T),
            loss = w c (sum over j of p_j log(p_j / q_{i_j}) + p_rest log(p_rest / q_rest)), q_rest the sum of q over the columns
            that are not listed, and dz, the gradient of its sum.  An entry with a column of -1 is none; a row without any has
            nothing to learn: zeros.
"""
from __future__ import annotations

import math

import torch

own = False             # True: the package's operators; False: the plain form

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 128
SCALE = 256.0           # the constant factor c of the distillation's loss: what keeps gradients in binary16's range


# ------------------------------------------------------------------ cases
def _quantise(rows, columns, mode, std=1.0):
    return {"op": "quantise", "rows": rows, "columns": columns, "mode": mode, "std": std}


def _product(rows, inputs, outputs, mode):
    return {"op": "product", "rows": rows, "columns": inputs, "outputs": outputs, "mode": mode}


def _top(rows, columns, k, mode, temperature=1.0, masked=0.0):
    return {"op": "top", "rows": rows, "columns": columns, "k": k, "mode": mode, "temperature": temperature, "masked": masked}


def _distill(what, rows, columns, k, mode, temperature=1.0, rest=True, masked=0.0):
    return {"op": "distill", "what": what, "rows": rows, "columns": columns, "k": k, "mode": mode, "temperature": temperature,
            "rest": rest, "masked": masked}


def listed():
    return [
        # the input of a product while answering a few requests: latency
        {"name": "quantise_tokens_bf16", **_quantise(8, 2048, "bf16")},
        # laying out the weights of a vocabulary's head once: the largest, an odd width
        {"name": "quantise_weights_f32", **_quantise(50021, 2001, "f32", 0.02)},
        # the teacher's next token through a large block's products: the weights are read once, latency counts
        {"name": "product_token_bf16", **_product(1, 4096, 11264, "bf16")},
        # a few requests at once over a vocabulary
        {"name": "product_batch_f16", **_product(24, 1600, 32768, "f16")},
        # some hundred tokens of uneven files through a block, sizes that divide by nothing
        {"name": "product_ragged_bf16", **_product(333, 2001, 4160, "bf16")},
        # a whole batch of tokens: the largest
        {"name": "product_prompt_bf16", **_product(8192, 4096, 11264, "bf16")},
        # logits of the next tokens of a few requests, in 32 bits
        {"name": "top_tokens_f32", **_top(8, 32768, 40, "f32")},
        # the teacher's answers for a batch of tokens, an odd vocabulary with a padded end
        {"name": "top_batch_bf16", **_top(4096, 50021, 64, "bf16", 2.0, 0.01)},
        # a small vocabulary: many short rows
        {"name": "top_short_f16", **_top(14336, 1000, 8, "f16", 1.0)},
        # a small training step in 32 bits on a small vocabulary
        {"name": "distill_small_f32", **_distill("train", 320, 1001, 8, "f32", 1.0, False)},
        # a training step: 28 files (one per pair of 8 nodes) of 512 tokens
        {"name": "distill_train_bf16", **_distill("train", 14336, 32768, 64, "bf16", 2.0)},
        # a large odd vocabulary with a padded end: the loss and its gradient, rows that no 16 bytes divide
        {"name": "distill_large_f16", **_distill("train", 1500, 131071, 20, "f16", 1.5, True, 0.02)},
    ]


def draw(rng):
    """One more case of the same ranges: one row to 65536, vocabularies of 100 to 262144, products of one token to 8192.  None
    costs more than the largest listed one of its kind."""

    def size(low, high, grain=1):
        v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
        return max(1, v // grain) * grain

    while True:
        op = rng.choices(["quantise", "product", "top", "distill"], [1, 3, 2, 3])[0]
        mode, grain = rng.choice(["bf16", "bf16", "f16", "f32"]), rng.choice([1, 1, 8, 64])
        temperature, masked = rng.choice([0.7, 1.0, 2.0]), rng.choice([0.0, 0.0, 0.03])
        if op == "quantise":
            case = _quantise(size(1, 65536), size(64, 16384, grain), mode, rng.choice([0.02, 1.0]))
        elif op == "product":
            rows = size(1, 64) if rng.random() < 0.4 else size(1, 8192, rng.choice([1, 16, 128]))
            case = _product(rows, size(128, 11264, grain), size(128, 32768, grain), mode)
        elif op == "top":
            case = _top(size(1, 16384), size(100, 262144, grain), size(1, 128), mode, temperature, masked)
        else:
            case = _distill(rng.choice(["loss", "train", "train"]), size(1, 16384), size(100, 262144, grain), size(1, 128), mode,
                            temperature, rng.random() < 0.7, masked)
        values = case["rows"] * case["columns"]
        most = {"quantise": 50021 * 2001, "product": 1 << 40, "top": 4096 * 50021, "distill": 14336 * 32768}[op]
        need = work(case)
        if values <= most and need["flops"] <= 2 * 8192 * 4096 * 11264 and need["bytes"] <= 1.9e9:
            return case


def _padded(columns):
    """Columns of a row of 8-bit numbers, and bytes of its scales."""
    blocks = -(-columns // BLOCK)
    return blocks * BLOCK, -(-blocks // 4) * 4


def work(case):
    rows, columns, eb = case["rows"], case["columns"], BYTES[case["mode"]]
    if case["op"] == "quantise":
        return {"bytes": rows * (columns * eb + sum(_padded(columns))), "flops": 2 * rows * columns}
    if case["op"] == "product":
        n = case["outputs"]
        return {"bytes": (rows + n) * sum(_padded(columns)) + rows * n * eb, "flops": 2 * rows * n * columns}
    if case["op"] == "top":
        return {"bytes": rows * (columns * eb + 8 * case["k"] + 4), "flops": 4 * rows * columns}
    passes = 2 if case["what"] == "train" else 1           # z read, dz written
    return {"bytes": rows * (passes * columns * eb + 8 * case["k"] + 12), "flops": 6 * rows * columns}


# ------------------------------------------------------------------ inputs
def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype, rows, columns = TYPES[case["mode"]], case["rows"], case["columns"]

    def normal(*shape, std=1.0, mean=0.0):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, std, generator=g)

    if case["op"] == "quantise":
        # a few columns are much larger than the others, as activations have them
        loud = 1 + 30 * (torch.rand(columns, device="cuda", generator=g) < 0.01).float()
        return {"x": (normal(rows, columns, std=case["std"]) * loud).to(dtype)}
    if case["op"] == "product":
        s = {}
        for name, n, std in (("x", rows, 1.0), ("w", case["outputs"], 1 / math.sqrt(columns))):
            s["q" + name], s["s" + name] = _plain_quantise(normal(n, columns, std=std))
        return s
    valid = columns - int(columns * case["masked"])         # the padded end of a vocabulary is masked
    z = normal(rows, columns, std=2.0)
    if case["op"] == "distill":
        # the teacher's list: distinct columns (its entries are less than columns / k apart and do not wrap); the student has learned some
        k = min(case["k"], valid // 2)
        each = 1 + (torch.rand(rows, 1, device="cuda", generator=g) * (valid // k)).long().clamp(max=valid // k - 1)
        place = torch.argsort(torch.rand(rows, k, device="cuda", generator=g), 1)
        index = each * place + (torch.rand(rows, 1, device="cuda", generator=g) * (valid - each * (k - 1))).long()
        value = normal(rows, k, std=1.5, mean=5.0).sort(1, descending=True).values
        z.scatter_(1, index, 0.7 * value + normal(rows, k))
        s = {"index": index.int(), "value": value}
        short = torch.rand(rows, 1, device="cuda", generator=g) < 0.05             # rows whose list is shorter, or empty
        keep = (torch.rand(rows, 1, device="cuda", generator=g) * k).long()
        absent = short & (torch.arange(k, device="cuda") >= keep)
        s["index"].masked_fill_(absent, -1)
        s["value"].masked_fill_(absent, -math.inf)
        if k < case["k"]:
            s = {"index": torch.nn.functional.pad(s["index"], (0, case["k"] - k), value=-1),
                 "value": torch.nn.functional.pad(s["value"], (0, case["k"] - k), value=-math.inf)}
        s["rest"] = normal(rows, std=0.7, mean=4.0) if case["rest"] else None
        # padded tokens count for nothing
        s["weight"] = (torch.rand(rows, device="cuda", generator=g) > 0.03).float() * (0.5 + torch.rand(rows, device="cuda", generator=g))
    else:
        s = {}
    z[:, valid:] = -math.inf
    return {"z": z.to(dtype), **s}


def prepare(case, seed):
    """The inputs, the buffers that a program keeps for results, and the package's handle where that is what runs."""
    s = {"case": case, **_inputs(case, seed)}
    rows, columns, dtype = case["rows"], case["columns"], TYPES[case["mode"]]
    new = lambda dtype, *shape: torch.zeros(shape, dtype=dtype, device="cuda")  # noqa: E731
    if case["op"] == "quantise":
        wide, blocks = _padded(columns)
        s["q"], s["scale"] = new(torch.float8_e4m3fn, rows, wide), new(torch.uint8, rows, blocks)
    elif case["op"] == "product":
        s["y"] = new(dtype, rows, case["outputs"])
    elif case["op"] == "top":
        k = case["k"]
        s["index"], s["value"], s["rest"] = new(torch.int32, rows, k), new(torch.float32, rows, k), new(torch.float32, rows)
    else:
        s["loss"], s["dz"] = new(torch.float32, rows), new(dtype, rows, columns) if case["what"] == "train" else None
    s["block"] = _handle(case) if own else None
    return s


def _handle(case):
    import paper_1805_01993_amd as L
    return L.ccdc_block(64, 1, case["mode"]).bind([case["rows"]]).upload()


# ------------------------------------------------------------------ one pass
def run(state):
    if own:
        return _run_own(state)
    s, case = state, state["case"]
    if case["op"] == "quantise":
        q, scale = _plain_quantise(s["x"].float())
        return {"q": q, "scale": scale}
    if case["op"] == "product":
        return {"y": (_wide(s["qx"], s["sx"]) @ _wide(s["qw"], s["sw"]).t()).to(TYPES[case["mode"]])}
    return _plain_top(s) if case["op"] == "top" else _plain_distill(s)


def _run_own(s):
    case, block = s["case"], s["block"]
    if case["op"] == "quantise":
        block.quantise(s["x"], s["q"], s["scale"])
        return {"q": s["q"], "scale": s["scale"]}
    if case["op"] == "product":
        block.packed_product(s["qx"], s["sx"], s["qw"], s["sw"], s["y"])
        return {"y": s["y"]}
    if case["op"] == "top":
        block.top(s["z"], s["index"], s["value"], rest=s["rest"], temperature=case["temperature"])
        return {k: s[k] for k in ("index", "value", "rest")}
    block.distill(s["z"], s["index"], s["value"], s["loss"], s["dz"], rest=s["rest"], temperature=case["temperature"],
                  weight=s["weight"], scale=SCALE)
    return {"loss": s["loss"], "dz": s["dz"]} if case["what"] == "train" else {"loss": s["loss"]}


# ------------------------------------------------------------------ the plain form: elementary operations in 32 bits
def _plain_quantise(x):
    """q and the scales of a matrix in 32 bits.  Scales are powers of two, so that only the rounding to 8 bits rounds."""
    rows, columns = x.shape
    wide, kept = _padded(columns)
    blocks = torch.nn.functional.pad(x, (0, wide - columns)).view(rows, wide // BLOCK, BLOCK)
    most, power = torch.frexp(blocks.abs().amax(2))                           # max |x| = most 2^power, most in [1/2, 1); 448 = 7/8 2^9
    e = (power - 9 + (most > 0.875).int()).clamp(min=-127)
    e = torch.where(most == 0, 0, e)
    q = (blocks * _power(127 - e)[:, :, None]).to(torch.float8_e4m3fn).view(rows, wide)
    scale = torch.full((rows, kept), 127, dtype=torch.uint8, device=x.device)
    scale[:, :wide // BLOCK] = (e + 127).to(torch.uint8)
    return q, scale


def _power(scale):
    """2^(scale - 127) in 32 bits, for 0 to 254, by its bits: a power's rounding would change what is rounded to 8 bits."""
    scale = scale.int()
    return torch.where(scale > 0, scale << 23, 1 << 22).view(torch.float32)


def _wide(q, scale):
    """A matrix of 8-bit numbers in 32 bits."""
    rows, wide = q.shape
    return (q.float().view(rows, -1, BLOCK) * _power(scale[:, :wide // BLOCK])[:, :, None]).view(rows, wide)


def _lse(v):
    """log of the sum of exp over the last dimension; -inf where there is nothing."""
    m = v.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    return torch.log(torch.exp(v - m).sum(-1)) + m[..., 0]


def _plain_top(s):
    case, z = s["case"], s["z"].float()
    rows, columns = z.shape
    k = min(case["k"], columns)
    bits = (z + 0.0).view(torch.int32)                                        # (no negative zero)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long()                       # whole numbers in the order of the logits
    last = 0xFFFFFFFF - torch.arange(columns, device=z.device)                # of equal ones the lower column is the larger
    best = torch.topk((order << 32) + last, k, dim=1).values
    index = 0xFFFFFFFF - (best & 0xFFFFFFFF)
    value = z.gather(1, index)
    rest = _lse(z.scatter(1, index, -math.inf) / case["temperature"])
    out_index = torch.full((rows, case["k"]), -1, dtype=torch.int32, device=z.device)
    out_value = torch.full((rows, case["k"]), -math.inf, dtype=torch.float32, device=z.device)
    out_index[:, :k] = torch.where(value > -math.inf, index, -1).int()
    out_value[:, :k] = value
    return {"index": out_index, "value": out_value, "rest": rest}


def _plain_distill(s):
    case, T = s["case"], s["case"]["temperature"]
    z, index = s["z"].float() / T, s["index"].long()
    rows, columns = z.shape
    again = ((index[:, :, None] == index[:, None, :]).tril(-1)).any(2)        # a column that was listed before
    there = (index >= 0) & (index < columns) & ~again
    at = torch.where(there, index, 0)
    t = torch.where(there, s["value"] / T, -math.inf)
    if s["rest"] is not None:
        t = torch.cat((t, s["rest"][:, None]), 1)
    some = there.any(1)
    log_p = t - torch.where(some, _lse(t), 0.0)[:, None]
    p = torch.exp(log_p)
    member = torch.zeros(rows, columns + 1, dtype=torch.bool, device=z.device)
    member = member.scatter_(1, torch.where(there, index, columns), True)[:, :columns]
    lse, lse_rest = _lse(z), _lse(z.masked_fill(member, -math.inf))
    log_q = z.gather(1, at) - lse[:, None]
    if s["rest"] is not None:
        log_q = torch.cat((log_q, (lse_rest - lse)[:, None]), 1)
    weight = torch.where(some, s["weight"], 0.0) * SCALE
    loss = weight * torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1)
    out = {"loss": torch.where(weight == 0, 0.0, loss)}
    if case["what"] == "train":
        d = torch.exp(z - lse[:, None])
        if s["rest"] is not None:
            d = torch.where(member, d, d - p[:, -1:] * torch.exp(z - lse_rest[:, None]))
        d.scatter_add_(1, at, torch.where(there, -p[:, :index.shape[1]], 0.0))
        d = d * (weight / T)[:, None]
        out["dz"] = torch.where(weight[:, None] == 0, 0.0, d).to(s["z"].dtype)
    return out


# ------------------------------------------------------------------ the same from the definitions, in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "quantise":
        return _exact_quantise(s["x"].double())
    if case["op"] == "product":
        values = []
        for name in ("x", "w"):
            power = torch.repeat_interleave(s["s" + name].long() - 127, BLOCK, 1)[:, :s["q" + name].shape[1]]
            values.append(s["q" + name].double() * _exact_power(power))
        return {"y": values[0] @ values[1].t().contiguous()}
    z, T = s["z"].double(), case["temperature"]
    columns = z.shape[1]
    if case["op"] == "top":
        # a stable sort keeps the order of equal ones
        value, index = torch.sort(z, dim=1, descending=True, stable=True)
        k = min(case["k"], columns)
        rest = torch.logsumexp(value[:, k:] / T, 1) if k < columns else torch.full_like(value[:, 0], -math.inf)
        pad = (0, case["k"] - k)
        index = torch.where(value[:, :k] > -math.inf, index[:, :k], -1)
        return {"index": torch.nn.functional.pad(index, pad, value=-1).int(),
                "value": torch.nn.functional.pad(value[:, :k], pad, value=-math.inf), "rest": rest}

    # each row as a distribution over its listed columns and all others, differentiated
    index, k = s["index"].long(), case["k"]
    there = index >= 0
    row = torch.arange(len(z), device=z.device)[:, None].expand_as(index)
    groups = torch.full((len(z), columns), k, dtype=torch.int64, device=z.device)
    groups[row[there], index[there]] = torch.arange(k, device=z.device).expand_as(index)[there]
    teacher = s["value"].double() / T
    teacher = torch.cat((teacher, s["rest"].double()[:, None] if s["rest"] is not None else torch.full_like(teacher[:, :1], -math.inf)), 1)
    teacher = teacher.masked_fill(torch.cat((~there, torch.zeros_like(there[:, :1])), 1), -math.inf)
    learns = there.any(1)
    teacher[~learns] = 0.0
    p = torch.softmax(teacher, 1)
    z = z.requires_grad_(case["what"] == "train")
    log_q = torch.log_softmax(z / T, 1)
    listed = log_q.gather(1, torch.where(there, index, 0))
    others = torch.logsumexp(log_q.masked_fill(groups < k, -math.inf), 1)
    both = torch.cat((listed, others[:, None]), 1)
    both = torch.where(p > 0, both, 0.0)
    terms = p * (torch.where(p > 0, p, 1.0).log() - both)
    loss = terms.sum(1) * torch.where(learns, s["weight"].double() * SCALE, 0.0)
    if case["what"] != "train":
        return {"loss": loss}
    (dz,) = torch.autograd.grad(loss.sum(), z)
    return {"loss": loss.detach(), "dz": dz}


def _exact_power(e):
    """2^e in 64 bits, by its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_quantise(x):
    rows, columns = x.shape
    wide, kept = _padded(columns)
    blocks = torch.nn.functional.pad(x, (0, wide - columns)).view(rows, -1, BLOCK)
    most = blocks.abs().amax(2)
    e = torch.ceil(torch.log2(torch.where(most > 0, most, 448.0) / 448.0))
    # the logarithm may be off by its rounding next to a power of two
    e = torch.where(most > 448.0 * _exact_power(e), e + 1, e)
    e = torch.where((most > 0) & (most <= 448.0 * _exact_power(e - 1)), e - 1, e).clamp(min=-127)
    v = blocks * _exact_power(-e)[:, :, None]
    # e4m3: four significant bits, from 2^-6 down steps of 2^-9; to nearest, ties to even
    step = _exact_power(torch.frexp(v.abs().clamp(min=2.0 ** -6)).exponent - 4)
    scale = torch.full((rows, kept), 127, dtype=torch.uint8, device=x.device)
    scale[:, :wide // BLOCK] = (e + 127).to(torch.uint8)
    return {"q": (torch.round(v / step) * step).view(rows, wide), "scale": scale}
