"""AdamW over a tensor list and the global gradient norm in fp64 numpy, from the definition in include/dynbatch.h,
with elementwise bounds on what fp32 arithmetic may be off.  Shares nothing with the library."""
import math

import numpy as np

BLOCK = 256
EPS32 = 2.0**-24              # half a unit in the last place of binary32, relative


def f32(x):
    return float(np.float32(x))


def widen(g):
    """fp32 array, or uint16 bf16 bits, as fp64."""
    return (g.astype(np.uint32) << 16).view(np.float32).astype(np.float64) if g.dtype == np.uint16 else g.astype(np.float64)


def weights(b):
    return [np.float64(np.float32(x / sum(b))) for x in b]


def aggregate(grads, b):
    """(g, bound): the weighted sum of the workers that have samples, and what fp32 may be off: a product is rounded, then
    the sums of its group of four (three at most), then the groups' sums (one for each four workers), so that n workers'
    products are rounded n times at most (a single worker's weight is 1), each time by 2^-24 of the sum of magnitudes."""
    act = [(w, widen(g)) for w, g, n in zip(weights(b), grads, b) if n > 0]
    g = sum(w * x for w, x in act)
    size = sum(w * np.abs(x) for w, x in act)
    return g, len(act) * EPS32 * 1.01 * size + 2.0**-149


def norm(tensors, b):
    return math.sqrt(sum(float(np.sum(aggregate(g, b)[0] ** 2)) for g in tensors))


# ---- 8-bit moments ------------------------------------------------------------------------------
def e4m3_values(codes):
    """uint8 e4m3 codes as fp64 values."""
    c = codes.astype(np.int64)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e == 0, f * 2.0**-9, (8 + f) * 2.0 ** (e - 10.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


def random_bits(position, seed, step):
    mask = 2**64 - 1
    z = (seed + 0x9E3779B97F4A7C15 * step) & mask
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & mask
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & mask
    z ^= z >> 31
    low = np.uint64(0xFFFFFFFF)

    def fold(x, m):
        w = x * np.uint64(m)
        return ((w >> np.uint64(32)) ^ w) & low

    s = position.astype(np.uint64)
    x = fold((s & low) ^ np.uint64(z & 0xFFFFFFFF), 0xAC4C1B51)
    x ^= np.uint64(z >> 32) ^ (((s >> np.uint64(32)) * np.uint64(0x85EBCA6B)) & low)
    return fold(x, 0xD6E8FEB5)


def round_up_by_chance(y, chance):
    """Magnitude of the code for y >= 0 with 16 random bits: monotone in y."""
    e = np.floor(np.log2(np.maximum(y, 2.0**-40)))
    e = np.where(2.0**e > y, e - 1, e)
    q = 2.0 ** (np.maximum(e, -6.0) - 3)
    return np.minimum(q * np.floor(y / q + chance / 65536.0), 448.0)


def block_max(x):
    n = x.size
    pad = np.zeros(-(-n // BLOCK) * BLOCK)
    pad[:n] = np.abs(x)
    return np.maximum(pad.reshape(-1, BLOCK).max(1), 2.0**-100)


def code_range(x, off, position, seed, step, second):
    """(lowest, highest) magnitude the code may have, and (scale, its bound): |x - computed x| <= off."""
    top = block_max(x)
    top_off = block_max(off) + 2 * EPS32 * top
    each = lambda v: np.repeat(v, BLOCK)[:x.size]  # noqa: E731
    r = random_bits(position + np.arange(x.size), seed, step)
    chance = (r >> np.uint64(16) if second else r & np.uint64(0xFFFF)).astype(np.float64)
    y = np.abs(x) * 448 / each(top)
    y_off = off * 448 / each(top) + y * (each(top_off / top) + 4 * EPS32) + 2.0**-29      # subnormal y: 2^-149 2^120
    lo, hi = round_up_by_chance(np.maximum(y - y_off, 0), chance), round_up_by_chance(y + y_off, chance)
    if second:
        # the lowest code is for values that come out above zero: a gradient that cancels to within its own rounding
        # (|h| <= its bound, e.g. 3 g_1 = -8 g_2 with weights 3/11 and 8/11) may be zero in one of fp32 and fp64 and not in the other
        lo, hi = np.where(x > off, np.maximum(lo, 2.0**-9), lo), np.where(x + off > 0, np.maximum(hi, 2.0**-9), hi)
    return lo, hi, top / 448, top_off / 448 + 2 * EPS32 * top / 448


# ---- one step of one tensor -----------------------------------------------------------------------
def step(grads, b, p, m, u, lr, beta1, beta2, eps, t, wd=0.0, factor=1.0, factor_off=0.0):
    """New (p, m, u) of one tensor and bounds for each: inputs fp64 (the values the kernel starts from)."""
    lr, beta1, beta2, eps, wd = f32(lr), f32(beta1), f32(beta2), f32(eps), f32(wd)
    g, g_off = aggregate(grads, b)
    h = factor * g
    h_off = factor * g_off + (factor_off + 2 * EPS32) * np.abs(h)
    m1 = beta1 * m + (1 - beta1) * h
    m_off = (1 - beta1) * h_off + 3 * EPS32 * (np.abs(beta1 * m) + np.abs((1 - beta1) * h)) + 2.0**-147
    u1 = beta2 * u + (1 - beta2) * h * h
    u_off = (1 - beta2) * (2 * np.abs(h) + h_off) * h_off + 4 * EPS32 * u1 + 2.0**-147
    c1, c2 = 1 - beta1**t, 1 - beta2**t
    root = np.sqrt(u1)
    with np.errstate(divide="ignore", invalid="ignore"):
        root_off = np.minimum(np.sqrt(u_off), np.where(root > 0, u_off / root, np.inf)) + 2 * EPS32 * root
        d = root / math.sqrt(c2) + eps
        d_off = root_off / math.sqrt(c2) + 3 * EPS32 * d
        least = np.maximum(d - d_off, eps * (1 - 3 * EPS32))
        move = lr / c1 * np.where(m1 == 0, 0.0, m1 / d)
        move_off = lr / c1 * (m_off / least + np.abs(m1) * d_off / (d * least)) + 5 * EPS32 * np.abs(move)
    p1 = p * (1 - lr * wd) - move
    p_off = move_off + 3 * EPS32 * np.abs(p) + 2 * EPS32 * np.abs(p1)
    return (p1, m1, u1), (p_off, m_off, u_off)
