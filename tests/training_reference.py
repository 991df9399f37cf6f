"""The training step's operators in 64 bits on the CPU, from their definitions, with none of the library's code."""
import math

import torch


def exponents(x, rows_per):
    """Exponent bytes [ceil(rows / rows_per)][ceil(cols / 128)] of a matrix: the least E >= 10 with the block's largest finite magnitude
    <= 448 * 2^(E - 127)."""
    x = x.double()
    a = torch.where(torch.isfinite(x), x.abs(), 0.0)
    a = torch.nn.functional.pad(a, (0, -a.shape[1] % 128, 0, -a.shape[0] % rows_per))
    a = a.view(a.shape[0] // rows_per, rows_per, a.shape[1] // 128, 128).amax(dim=(1, 3))
    e = torch.full(a.shape, 10, dtype=torch.int64)
    for _ in range(256):                     # one step at a time: no logarithm whose rounding could matter
        e += (a > 448.0 * torch.exp2(e.double() - 127)).long()
    return e


def spread(e, rows_per, rows, cols):
    return e.repeat_interleave(rows_per, 0)[:rows].repeat_interleave(128, 1)[:, :cols]


NUMBERS = torch.tensor([(m if k == 0 else 8 + m) * 2.0 ** (max(k, 1) - 10) for k in range(16) for m in range(8)][:127], dtype=torch.float64)


def codes(x, rows_per):
    """(codes of the existing elements, exponents); a NaN's code is 127 whatever its sign."""
    e = exponents(x, rows_per)
    t = x.double() * torch.exp2(127 - spread(e, rows_per, *x.shape).double())
    size = t.abs().nan_to_num(0.0, 0.0, 0.0)
    up = torch.searchsorted(NUMBERS, size).clamp(max=126)             # first number >= size
    down = (up - 1).clamp(min=0)
    over, under = NUMBERS[up] - size, size - NUMBERS[down]
    c = torch.where((over < under) | ((over == under) & (up % 2 == 0)), up, down)
    c = torch.where(size == 0, 0, c) + 128 * torch.signbit(t).long()
    return torch.where(torch.isfinite(x.double()), c, 127), e


def values(c, e, rows_per, cols):
    c = c[:, :cols].long()
    v = torch.cat([NUMBERS, torch.tensor([math.nan], dtype=torch.float64)])[c & 127]
    return torch.where(c > 127, -v, v) * torch.exp2(spread(e.long(), rows_per, c.shape[0], cols).double() - 127)


def blocks_values(b):
    """Values of a Blocks, in fp64 on the CPU."""
    return values(b.codes.cpu(), b.exps.cpu()[:, :(b.cols + 127) // 128], 128 if b.tiles else 1, b.cols)


def kept(x):
    c, e = codes(x, 1)
    return values(c, e, 1, x.shape[1])


def layer_norm(x, gamma, beta, eps):
    x = x.double()
    mean = x.mean(1)
    rstd = (((x - mean[:, None]) ** 2).mean(1) + eps) ** -0.5
    h = (x - mean[:, None]) * rstd[:, None]
    return h * (1.0 if gamma is None else gamma.double()) + (0.0 if beta is None else beta.double()), mean, rstd


def layer_norm_grad(dy, x, gamma, mean, rstd):
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    h = (x - mean) * rstd
    q = dy if gamma is None else dy * gamma.double()
    return rstd * (q - q.mean(1, keepdim=True) - h * (q * h).mean(1, keepdim=True)), (dy * h).sum(0), dy.sum(0)


def act(kind, x):
    x = x.double()
    if kind == "relu":
        return torch.where(x < 0, 0.0, x)
    if kind == "silu":
        return x / (1 + torch.exp(-x))
    return x * 0.5 * torch.erfc(-x / math.sqrt(2))


def act_slope(kind, x):
    x = x.double()
    if kind == "relu":
        return (x > 0).double()
    if kind == "silu":
        p = 1 / (1 + torch.exp(-x))
        return p * (1 + x * (1 - p))
    return 0.5 * torch.erfc(-x / math.sqrt(2)) + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
