"""Rows kept in 8 bits, by the definition and in 64 bits: what the tests of the calls that keep and take them compare with."""
import torch

FORMS = ("i8", "e4m3")
LARGEST = {"i8": 127.0, "e4m3": 448.0}
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


def e4m3(byte):
    """The number that a byte of e4m3 is."""
    sign, exponent, fraction = -1.0 if byte & 128 else 1.0, byte >> 3 & 15, byte & 7
    if byte & 127 == 127:
        return float("nan")
    return sign * (fraction / 8.0 * 2.0 ** -6 if exponent == 0 else (1 + fraction / 8.0) * 2.0 ** (exponent - 7))


def decoded(values, scales, width, form):
    """[N, width] in 64 bits on the CPU."""
    table = torch.tensor([float(b - 256 if b > 127 else b) if form == "i8" else e4m3(b) for b in range(256)], dtype=torch.float64)
    scale = torch.tensor([2.0 ** (b - 127) if b < 255 else float("nan") for b in range(256)], dtype=torch.float64)
    codes = table[values.cpu().long()].view(values.shape[0], values.shape[1] // 32, 32)
    return (codes * scale[scales.cpu().long()][:, :, None]).flatten(1)[:, :width]


def encoded(rows, form):
    """(codes' numbers [N, groups, 32], scales [N, groups, 1]) in 64 bits of rows in 64 bits: the least scale, from 2^-127, with which the largest of a group rounds to a code."""
    rows = rows.double().cpu()
    rows = torch.nn.functional.pad(rows, (0, -rows.shape[1] % 32)).unflatten(1, (-1, 32))
    top = rows.abs().amax(2, keepdim=True)
    exponent = torch.full(top.shape, -127.0, dtype=torch.float64)
    limit = 127.5 if form == "i8" else 448.0
    for e in range(-126, 128):
        short = top / 2.0 ** (e - 1)
        exponent = torch.where((short >= limit) if form == "i8" else (short > limit), float(e), exponent)
    scale = torch.exp2(exponent)
    return rounded(rows / scale, form), scale


def rounded(q, form):
    """To the nearest code, ties to even."""
    if form == "i8":
        return torch.round(q)
    step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
    step = torch.where(q.abs() < 2.0 ** -6, 2.0 ** -9, step)
    return torch.round(q / step) * step
