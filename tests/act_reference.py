"""Plain 64-bit forms of the activation operators for the tests (no code of the package)."""
import math

import torch

GROUP = 32
SILU, GELU_TANH, RELU = 0, 1, 2
INT8, E4M3, BF16 = 0, 1, 2


def encode(x, fmt):
    """(element values, scale bytes) of a [rows, cols] tensor: [rows, groups, 32] float64 on the element grid (INT8: multiples of 1/64),
    [rows, groups] int64.  A group with a value that is not finite: zeros and 255."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x.double(), (0, -cols % GROUP)).view(rows, -1, GROUP)
    finite = torch.isfinite(x).all(-1)
    x = torch.where(finite.unsqueeze(-1), x, 0.0)
    top = x.abs().amax(-1)
    exponent = torch.where(top > 0, torch.frexp(top).exponent.long() + 126, 0).clamp(min=0)   # biased; subnormals of FP32 have 0
    byte = (exponent - (8 if fmt == E4M3 else 0)).clamp(min=0)
    y = x * torch.exp2((127 - byte).double()).unsqueeze(-1)
    if fmt == INT8:
        y = torch.round(y * 64).clamp(-127, 127) / 64
    else:
        e = (torch.frexp(y).exponent.long() - 1).clamp(min=-6)
        step = torch.exp2((e - 3).double())
        y = (torch.round(y / step) * step).clamp(-448, 448)
    return y, torch.where(finite, byte, 255)


def values(element, byte, cols):
    """What a checkpoint stands for, in 64 bits."""
    v = element * torch.exp2((byte - 127).double()).unsqueeze(-1)
    v = torch.where((byte == 255).unsqueeze(-1), math.nan, v)
    return v.flatten(1)[:, :cols]


def elements_of(codes, fmt):
    """uint8 codes -> float64 element values."""
    if fmt == INT8:
        return codes.view(torch.int8).double() / 64
    c = codes.to(torch.int64)
    e, m = (c >> 3) & 15, c & 7
    mag = torch.where(e == 0, m.double() / 8 * 2.0 ** -6, (1 + m.double() / 8) * torch.exp2((e - 7).double()))
    return torch.where(c >= 128, -mag, mag)


def decode(act8):
    """The values of a package checkpoint in 64 bits, from its bytes alone."""
    rows, cols = act8.shape
    groups = -(-cols // GROUP)
    codes = act8.buffer[:rows * groups * GROUP].view(rows, groups, GROUP)
    first = -(-rows * groups * GROUP // 256) * 256
    byte = act8.buffer[first:first + rows * groups].view(rows, groups).long()
    return values(elements_of(codes, act8.fmt), byte, cols)


def act(g, kind):
    """(act(g), act'(g)) in the precision of g."""
    if kind == RELU:
        return torch.where(g < 0, 0.0, g), (g > 0).to(g.dtype)
    if kind == SILU:
        z, dz = g, torch.ones_like(g)
    else:
        c = 2 * math.sqrt(2 / math.pi)
        z, dz = c * (g + 0.044715 * g ** 3), c * (1 + 3 * 0.044715 * g ** 2)
    s = torch.special.expit(z)
    return g * s, s + g * s * (1 - s) * dz
