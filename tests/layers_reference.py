"""Layers, 8-bit checkpoints and the embedding table in 64 bits on the CPU, from their definitions, and the error bounds
that the GPU tests use."""
import math

import torch

GROUP = 32
BF16 = 2.0**-8       # half a step of bf16, relative
ADD = 2.0**-23       # one addition into the tensor cores' fp32 accumulator, which truncates


def act(z, name):
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "gelu":
        return z * torch.special.ndtr(z)
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(z, name):
    if name == "relu":
        return torch.where(z <= 0, torch.zeros_like(z), torch.ones_like(z))
    if name == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    return torch.ones_like(z)


def pack(x):
    """(codes float8_e4m3fn, scale bytes uint8) of x [rows, cols], value by value from the definition."""
    rows, cols = x.shape
    groups = -(-cols // GROUP)
    full = torch.zeros(rows, groups * GROUP, dtype=torch.float64)
    full[:, :cols] = x.double()
    full = full.view(rows, groups, GROUP)
    top = torch.where(torch.isfinite(full), full.abs(), torch.zeros_like(full)).amax(2)
    power = torch.full_like(top, -127.0)
    while True:                                             # the smallest power that is large enough
        short = top > 448 * torch.exp2(power)
        if not short.any():
            break
        power[short] += 1
    y = full / torch.exp2(power)[:, :, None]
    y = torch.where((power[:, :, None] == 120) & torch.isfinite(y), y.clamp(-240, 240), y)   # 256 * 2^120 is past fp32's end
    codes = y.to(torch.float32).to(torch.float8_e4m3fn)     # y has at most 24 bits; to nearest, ties to even
    nan = torch.full((), float("nan")).to(torch.float8_e4m3fn)
    codes = torch.where(torch.isfinite(full), codes.view(torch.uint8), nan.view(torch.uint8)).view(torch.float8_e4m3fn)
    return codes.view(rows, -1)[:, :cols].contiguous(), (power + 127).to(torch.uint8)


def unpack(codes, scale_bytes):
    """float64 values; a scale byte of 255 stands for NaN."""
    s = torch.exp2(scale_bytes.double() - 127)
    s[scale_bytes == 255] = float("nan")
    return codes.to(torch.float32).double() * s.repeat_interleave(GROUP, 1)[:, :codes.shape[1]]


def product_bound(a, b, extra=0.0):
    """Largest error of sum_k a(m,k) b(k,n) in the tensor cores' arithmetic: products are exact, 16 of them are added into
    the accumulator at a time; four more additions stand for the joining of a split reduction.  `extra`: relative error
    that the operands bring along."""
    return ((a.shape[1] / 16 + 4) * ADD + extra) * (a.abs() @ b.abs())


def embedding_grad(tokens, dy, vocab, scale):
    out = torch.zeros(vocab, dy.shape[1], dtype=torch.float64)
    for t, v in enumerate(tokens.tolist()):
        if 0 <= v < vocab:
            out[v] += dy[t].double()
    return out * scale
