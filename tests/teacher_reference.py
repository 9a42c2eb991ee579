"""The definitions of the calls that learn from a teacher (include/ccdc.h), in 64 bits, with how far fp32 sums and one rounding may be
from them."""
import math

import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}          # eps / 2, of a value at the lower end of its binade
SMALLEST = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}
U = 2.0 ** -24                                    # of a rounding in fp32


def power(e):
    """2^e in 64 bits, e a tensor of whole numbers."""
    return ((e.long() + 1023) << 52).view(torch.float64)


# every number of 8 bits (e4m3), by its bits
_bits = torch.arange(256)
_e, _m = _bits >> 3 & 15, (_bits & 7).double()
E4M3 = torch.where(_e > 0, (1 + _m / 8) * power(_e - 7), _m * 2.0 ** -9)
E4M3 = torch.where((_bits & 127) == 127, math.nan, torch.where(_bits >= 128, -E4M3, E4M3))


def quantise(x):
    """(bits [rows][padded], scales [rows][kept]) of a matrix in 64 bits."""
    rows, columns = x.shape
    blocks = -(-columns // 128)
    v = torch.zeros(rows, blocks * 128, dtype=torch.float64)
    v[:, :columns] = x.double().cpu()
    v = v.view(rows, blocks, 128)
    most = torch.where(torch.isfinite(v), v.abs(), 0.0).amax(2)
    e = torch.full(most.shape, -127)
    for step in range(-127, 129):                 # the least whole number with most <= 448 2^e
        e = torch.where(most > 448.0 * 2.0 ** (step - 1), step, e)
    e = torch.where(most == 0, 0, e.clamp(min=-127))
    v = v * power(-e)[:, :, None]
    # the nearest of all finite numbers, ties to the even one
    table, order = torch.sort(E4M3[:127])
    at = torch.searchsorted(table, v.abs().nan_to_num(0.0, posinf=0.0)).clamp(1, 126)
    low, high = table[at - 1], table[at]
    a = v.abs()
    take_high = (a - low > high - a) | ((a - low == high - a) & (order[at] % 2 == 0))
    bits = torch.where(take_high, order[at], order[at - 1])
    bits = torch.where(torch.isfinite(v), bits, 127) + 128 * torch.signbit(v)
    scale = torch.full((rows, -(-blocks // 4) * 4), 127)
    scale[:, :blocks] = e + 127
    return bits.view(rows, blocks * 128).to(torch.uint8), scale.to(torch.uint8)


def values(bits, scale):
    """What a packed matrix stands for."""
    blocks = bits.shape[1] // 128
    e = scale[:, :blocks].cpu().long()
    v = E4M3[bits.cpu().long()].view(len(bits), blocks, 128) * power(e - 127)[:, :, None]
    return torch.where((e == 255)[:, :, None], math.nan, v).view(len(bits), -1)


def product(x, w, mode):
    """x w' of two matrices of values, and how far a result may be off: sums in fp32; in the 16-bit modes what the instructions
    drop, up to 2^-13 of the largest of eight products for each of the other seven; one rounding."""
    y, size = x @ w.t(), x.abs() @ w.abs().t()
    off = x.shape[1] * U * size
    if mode != "f32":
        for first in range(0, x.shape[1], 8):
            group = (x[:, None, first:first + 8] * w[None, :, first:first + 8]).abs().amax(2)
            off = off + 7 * 2.0 ** -13 * group
    return y, off + HALF_STEP[mode] * (y.abs() + off) + SMALLEST[mode]


def top(z, k, temperature):
    """index, value, rest of rows of logits."""
    z = z.double().cpu()
    rows, columns = z.shape
    key = torch.where(z > -math.inf, z, -math.inf)             # NaNs too are not listed
    value, index = torch.sort(key, dim=1, descending=True, stable=True)
    out_index, out_value = torch.full((rows, k), -1, dtype=torch.int32), torch.full((rows, k), -math.inf, dtype=torch.float64)
    n = min(k, columns)
    listed = value[:, :n] > -math.inf
    out_index[:, :n] = torch.where(listed, index[:, :n], -1).int()
    out_value[:, :n] = value[:, :n]
    rest = z.clone().scatter_(1, index[:, :n], torch.where(listed, -math.inf, z.gather(1, index[:, :n])))
    return out_index, out_value, torch.logsumexp(rest / temperature, 1)


def distill(z, index, value, rest, temperature, weight, scale):
    """(loss, dz, and how far each may be off) of rows of logits, entry by entry of the definition."""
    z = z.double().cpu()
    rows, columns = z.shape
    loss, dz = torch.zeros(rows, dtype=torch.float64), torch.zeros(rows, columns, dtype=torch.float64)
    off_loss, off_dz = torch.zeros_like(loss), torch.zeros_like(dz)
    for r in range(rows):
        w = float(weight[r]) if weight is not None else 1.0
        listed, teacher = [], []
        for i, t in zip(index[r].tolist(), value[r].tolist()):
            if 0 <= i < columns and i not in listed:
                listed.append(i)
                teacher.append(t)
        row = z[r] / temperature
        if w == 0 or not listed or not bool((row != -math.inf).any()):
            continue
        others = torch.ones(columns, dtype=torch.bool)
        others[listed] = False
        t = torch.tensor([v / temperature for v in teacher] + [float(rest[r]) if rest is not None else -math.inf], dtype=torch.float64)
        if bool((t == -math.inf).all()):
            continue
        p = torch.softmax(t, 0)
        log_q = torch.log_softmax(row, 0)
        log_rest = torch.logsumexp(log_q[others], 0) if bool(others.any()) else torch.tensor(-math.inf, dtype=torch.float64)
        q = torch.cat((log_q[listed], log_rest[None]))
        some = ~(p == 0)
        terms = p[some] * (torch.log(p[some]) - q[some])
        c = w * scale
        loss[r] = c * terms.sum()
        g = torch.exp(log_q)
        of_rest = torch.zeros(columns, dtype=torch.float64)
        if p[-1] > 0 and log_rest > -math.inf:
            of_rest[others] = p[-1] * torch.exp(log_q[others] - log_rest)
        of_rest[listed] = p[:-1]
        dz[r] = c / temperature * (g - of_rest)
        # exponentials of x are some |x| U off (|x| is about log of the columns where they count), sums some hundred U; a term
        # p log q is as far off as it is large (with a masked column listed that is any size: three roundings of |log q|, each U |log q|)
        reach = 400 * U * (1 + row[row > -math.inf].abs().max().item() / 16)
        off_loss[r] = abs(c) * reach * (p[some] * (1 + torch.log(p[some]).abs() + q[some].abs())).sum()
        off_dz[r] = abs(c) / temperature * reach * (g + of_rest)
    return loss, dz, off_loss, off_dz
