"""AdamW over a list of tensors for K workers' batch-weighted gradients, with moments in 32 or in 8 bits, and the
global norm of the weighted gradient: cases, inputs, plain forms and 64-bit values.

A case describes one model's tensor list and one call:
  op      "adamw" or "norm"
  kind    how the list is built: "arena" (one tensor), "classifier" (weights and bias), "conv" (a residual
          convolution network), "decoder" (embedding, then per layer four square projections, two feed-forward
          matrices, their biases and two norms), "ragged" (sizes of no particular alignment)
  size, layers, vocab     its measures, by kind
  K, grad workers and the type of their gradients ("f32" or "bf16")
  shift   elements by which the workers' gradient buffers start off an aligned address
  state   32 or 8: bits of a moment's element (8: e4m3 with one fp32 scale for each 256 elements)
  copy    whether a bf16 working copy of the parameters is written along
  step    Adam's step count;  max_norm  the clipping bound (0: none);  beta2
Buffers are arenas in which every tensor starts at a multiple of 256 elements; what lies between is zero.
"""
import math
import random

import torch

own = False

BLOCK = 256
LR, BETA1, EPS, DECAY = 3e-4, 0.9, 1e-8, 0.1


def listed():
    return [
        # the norm alone, as a run logs it: three workers of a 1 Mi-parameter model, eight of a language model
        dict(name="norm 1Mi K3 f32", op="norm", kind="arena", size=1 << 20, layers=1, vocab=0, K=3, grad="f32", shift=0),
        dict(name="norm decoder 110M K16 bf16", op="norm", kind="decoder", size=1024, layers=8, vocab=8192, K=16,
             grad="bf16", shift=0),
        # the softmax classifier whose gradients the grouped worker call makes, clipped
        dict(name="w32 classifier 2M K4 f32 clip", op="adamw", kind="classifier", size=2048, layers=1, vocab=1000, K=4,
             grad="f32", shift=0, state=32, copy=False, step=10, max_norm=0.5, beta2=0.999),
        # a convolution network of 161 tensors, eight workers, no clipping
        dict(name="w32 conv 25M K8 f32", op="adamw", kind="conv", size=64, layers=16, vocab=1000, K=8, grad="f32", shift=0,
             state=32, copy=False, step=100, max_norm=0.0, beta2=0.999),
        # mixed precision: sixteen workers' bf16 gradients, fp32 parameters with a bf16 copy, clipped
        dict(name="w32 decoder 110M K16 clip", op="adamw", kind="decoder", size=1024, layers=8, vocab=8192, K=16,
             grad="bf16", shift=0, state=32, copy=True, step=1000, max_norm=1.0, beta2=0.95),
        # one gradient, already reduced: what the optimizer alone costs a larger model
        dict(name="w32 decoder 470M K1 bf16", op="adamw", kind="decoder", size=2048, layers=8, vocab=32000, K=1,
             grad="bf16", shift=0, state=32, copy=True, step=1000, max_norm=0.0, beta2=0.95),
        # the first step of a small model in 8 bits, where a call's latency is what it costs
        dict(name="w8 decoder 150K K2 f32", op="adamw", kind="decoder", size=64, layers=2, vocab=800, K=2, grad="f32",
             shift=0, state=8, copy=False, step=1, max_norm=0.0, beta2=0.999),
        # tensors of odd sizes, gradient buffers that start one element off
        dict(name="w8 ragged 5M K3 f32 shifted", op="adamw", kind="ragged", size=60013, layers=83, vocab=0, K=3, grad="f32",
             shift=1, state=8, copy=True, step=7, max_norm=0.0, beta2=0.999),
        dict(name="w8 decoder 110M K8 bf16", op="adamw", kind="decoder", size=1024, layers=8, vocab=8192, K=8,
             grad="bf16", shift=0, state=8, copy=True, step=1000, max_norm=0.0, beta2=0.95),
        # 8-bit states where they matter most: a larger model, one bf16 gradient, clipped
        dict(name="w8 decoder 470M K1 clip", op="adamw", kind="decoder", size=2048, layers=8, vocab=32000, K=1,
             grad="bf16", shift=0, state=8, copy=True, step=1000, max_norm=1.0, beta2=0.95),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    op = rng.choice(["norm", "adamw", "adamw", "adamw"])
    kind = rng.choice(["arena", "classifier", "conv", "decoder", "decoder", "ragged"])
    size, layers, vocab = {
        "arena": lambda: (log(5000, 64 << 20), 1, 0),
        "classifier": lambda: (log(50, 5000), 1, log(2, 5000)),
        "conv": lambda: (log(8, 100), rng.randint(4, 24), log(10, 1000)),
        "decoder": lambda: (log(30, 1300), rng.randint(1, 10), log(200, 20000)),
        "ragged": lambda: (log(500, 300000), rng.randint(2, 120), 0),
    }[kind]()
    c = dict(op=op, kind=kind, size=size, layers=layers, vocab=vocab)
    n = sum(math.prod(s) for s in shapes(c))
    c["K"] = max(1, min(log(1, 24), int(1.6e9 // n)))
    c["grad"] = rng.choice(["f32", "bf16"])
    c["shift"] = rng.choice([0, 0, 0, 1, 3])
    if op == "adamw":
        c.update(state=rng.choice([32, 8]), copy=rng.random() < 0.5, step=log(1, 100000),
                 max_norm=rng.choice([0.0, 0.25, 1.0]), beta2=rng.choice([0.95, 0.999]))
    return c


def shapes(case):
    """The tensors of the case's model, in order."""
    kind, s, layers, vocab = case["kind"], case["size"], case["layers"], case["vocab"]
    if kind == "arena":
        return [(s,)]
    if kind == "classifier":
        return [(s, vocab), (vocab,)]
    if kind == "ragged":
        rng = random.Random(1000 * s + layers)
        return [(rng.randint(1, 2 * s - 1),) for _ in range(layers)]
    if kind == "decoder":
        got = [(vocab, s)]
        for _ in range(layers):
            got += 4 * [(s, s), (s,)] + [(s,), (s,), (4 * s, s), (4 * s,), (s, 4 * s), (s,), (s,), (s,)]
        return got + [(s,), (s,)]
    # conv: a 7x7 stem, `layers` bottleneck blocks in four stages (3 : 4 : 6 : 3), each convolution with scale and shift
    per = [max(1, round(layers * r / 16)) for r in (3, 4, 6, 3)]
    got, width = [(s, 3, 7, 7), (s,), (s,)], s
    for stage, blocks in enumerate(per):
        mid = s << stage
        for blk in range(blocks):
            got += [(mid, width, 1, 1), (mid,), (mid,), (mid, mid, 3, 3), (mid,), (mid,), (4 * mid, mid, 1, 1), (4 * mid,), (4 * mid,)]
            if blk == 0:
                got += [(4 * mid, width, 1, 1), (4 * mid,), (4 * mid,)]
            width = 4 * mid
    return got + [(vocab, width), (vocab,)]


def _layout(case):
    """Element counts, arena offsets and arena length."""
    sizes = [math.prod(s) for s in shapes(case)]
    starts, at = [], 0
    for n in sizes:
        starts.append(at)
        at += -(-n // BLOCK) * BLOCK
    return sizes, starts, at


def work(case):
    n = sum(_layout(case)[0])
    g = 4 if case["grad"] == "f32" else 2
    if case["op"] == "norm":
        return {"bytes": n * case["K"] * g + 4, "flops": n * (2 * case["K"] + 2)}
    moments = 16 if case["state"] == 32 else 4 + 16 / BLOCK
    return {"bytes": n * (case["K"] * g + 8 + moments + (2 if case["copy"] else 0)),
            "flops": n * (2 * case["K"] + (16 if case["state"] == 32 else 40))}


def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    sizes, starts, total = _layout(case)
    K, adamw = case["K"], case["op"] == "adamw"
    blocks = torch.tensor([-(-n // BLOCK) for n in sizes], device=dev)
    # which elements of the arena belong to a tensor, and each tensor's own gradient scale (layers differ)
    owner = torch.repeat_interleave(torch.arange(len(sizes), device=dev), blocks)
    left = (torch.tensor(sizes, device=dev) + torch.tensor(starts, device=dev))[owner] - torch.arange(0, total, BLOCK, device=dev)
    live = torch.arange(BLOCK, device=dev)[None, :] < left[:, None]
    spread = torch.exp(torch.empty(len(sizes), device=dev).normal_(0.0, 1.0, generator=gen))[owner][:, None]
    normal = lambda std: torch.empty(total, device=dev).normal_(0.0, std, generator=gen)  # noqa: E731
    dtype = torch.float32 if case["grad"] == "f32" else torch.bfloat16
    row = -(-(total + case["shift"]) // BLOCK) * BLOCK
    grads = torch.zeros(K, row, dtype=dtype, device=dev)[:, case["shift"]:case["shift"] + total]
    for k in range(K):
        grads[k].copy_((normal(1e-3).view(-1, BLOCK) * spread * live).view(-1))
    rng = random.Random(seed)
    state = {"case": case, "grads": grads, "batches": [rng.randint(8, 256) for _ in range(K)], "seed": rng.getrandbits(62),
             "norm": torch.zeros(1, device=dev)}
    views = lambda t: [t[s:s + n] for s, n in zip(starts, sizes)]  # noqa: E731
    if adamw:
        state["params"] = (normal(0.02).view(-1, BLOCK) * live).view(-1)
        first = (normal(3e-4).view(-1, BLOCK) * spread * live).view(-1)
        # a running mean of squares: spread about the gradient's variance, not down to zero
        second = ((normal(1e-3).view(-1, BLOCK).square() + 2e-7) * spread.square() * live * 0.5).view(-1)
        if case["step"] == 1:
            first.zero_(), second.zero_()
        decays = [DECAY if len(s) > 1 else 0.0 for s in shapes(case)]
        state["decay"] = torch.tensor(decays, device=dev)[owner][:, None]
        if case["state"] == 32:
            state["first"], state["second"] = first, second
        else:
            for name, x in (("first", first.view(-1, BLOCK)), ("second", second.view(-1, BLOCK))):
                scale = x.abs().amax(1) / 448
                codes = (x / scale.clamp_min(1e-30)[:, None]).clamp(-448, 448)
                if name == "second":  # a mean of squares that is not zero is not held as zero
                    codes = torch.where(x > 0, codes.clamp_min(2.0**-9), codes)
                codes = codes.to(torch.float8_e4m3fn)
                state[name], state[name + "_scale"] = codes.view(-1), scale
        if case["copy"]:
            state["working"] = state["params"].to(torch.bfloat16)
    if own:
        # the handle that a program keeps beside its buffers
        from paper_2305_12213_b200 import binding
        lists = {"params": views(state["params"])} if adamw else {}
        if adamw:
            lists.update(first_moment=views(state["first"]), second_moment=views(state["second"]), weight_decay=decays,
                         clip=case["max_norm"] > 0)
            if case["copy"]:
                lists["params_bf16"] = views(state["working"])
            if case["state"] == 8:
                cut = lambda t: [t[s // BLOCK:s // BLOCK + -(-n // BLOCK)] for s, n in zip(starts, sizes)]  # noqa: E731
                lists.update(first_scale=cut(state["first_scale"]), second_scale=cut(state["second_scale"]))
        per_worker = [views(grads[k]) for k in range(K)]
        state["plan"] = binding.AdamWPlan(per_worker, **lists) if adamw else binding.GradNormPlan(per_worker)
    return state


def _outputs(state):
    case = state["case"]
    if case["op"] == "norm":
        return {"norm": state["norm"]}
    names = ["params", "first", "second"] + (["first_scale", "second_scale"] if case["state"] == 8 else [])
    names += (["working"] if case["copy"] else []) + (["norm"] if case["max_norm"] > 0 else [])
    return {name: state[name] for name in names}


def _random_bits(n, seed, step, device):
    """32 bits for each position 0 .. n - 1: two rounds of multiply and fold, keyed by the seed and the step."""
    z = (seed + 0x9E3779B97F4A7C15 * step) & (2**64 - 1)
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & (2**64 - 1)
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & (2**64 - 1)
    z ^= z >> 31
    low = 0xFFFFFFFF
    s = torch.arange(n, device=device)
    x = ((s & low) ^ (z & low)) * 0xAC4C1B51
    x = ((x >> 32) ^ x ^ (z >> 32) ^ ((s >> 32) * 0x85EBCA6B)) & low
    x = x * 0xD6E8FEB5
    return ((x >> 32) ^ x) & low


def _to_8_bits(x, bits, positive):
    """Codes and scales of blocks x [B, 256]: e4m3 steps below |x| 448 / max, taken up by chance with 16 random bits."""
    top = x.abs().amax(1, keepdim=True).clamp_min(2.0**-100)
    y = x.abs().double() * 448 / top.double()
    step = torch.exp2(torch.frexp(y.clamp_min(2.0**-6))[1].double() - 4)
    y = (torch.floor(y / step + bits / 65536) * step).clamp_max(448)
    if positive:
        y = torch.where(x > 0, y.clamp_min(2.0**-9), y)
    return torch.copysign(y, x).float().to(torch.float8_e4m3fn).view(-1), (top / 448).view(-1)


def run(state):
    case = state["case"]
    adamw = case["op"] == "adamw"
    if own:
        if adamw:
            state["plan"].step(state["batches"], LR, BETA1, case["beta2"], EPS, case["step"], max_norm=case["max_norm"],
                               seed=state["seed"], grad_norm=state["norm"] if case["max_norm"] > 0 else None)
        else:
            state["plan"].run(state["batches"], state["norm"])
        return _outputs(state)
    grads = state["grads"]
    weights = torch.tensor(state["batches"], dtype=torch.float64)
    weights = (weights / weights.sum()).float().to(grads.device)
    g = (weights[:, None] * grads).sum(0)
    if not adamw or case["max_norm"] > 0:
        norm = g.double().square().sum().sqrt()
        state["norm"].copy_(norm)
    if not adamw:
        return _outputs(state)
    if case["max_norm"] > 0:
        g = g * torch.clamp_max(case["max_norm"] / norm, 1.0).float()
    beta1, beta2 = (torch.tensor(b, dtype=torch.float32).item() for b in (BETA1, case["beta2"]))
    g, p = g.view(-1, BLOCK), state["params"].view(-1, BLOCK)
    m, u = state["first"].view(-1, BLOCK).float(), state["second"].view(-1, BLOCK).float()
    if case["state"] == 8:
        m, u = m * state["first_scale"][:, None], u * state["second_scale"][:, None]
    m = m * beta1 + g * (1 - beta1)
    u = u * beta2 + g * g * (1 - beta2)
    c1, c2 = 1 - beta1 ** case["step"], 1 - beta2 ** case["step"]
    p.copy_(p * (1 - LR * state["decay"]) - LR / c1 * m / ((u / c2).sqrt() + EPS))
    if case["copy"]:
        state["working"].copy_(state["params"])
    if case["state"] == 32:
        state["first"].copy_(m.view(-1)), state["second"].copy_(u.view(-1))
    else:
        bits = _random_bits(p.numel(), state["seed"], case["step"], p.device).view(-1, BLOCK)
        for name, x, r in (("first", m, bits & 0xFFFF), ("second", u, bits >> 16)):
            codes, scale = _to_8_bits(x, r, name == "second")
            state[name].copy_(codes), state[name + "_scale"].copy_(scale)
    return _outputs(state)


# ---------------------------------------------------------------------------------------------------------------
# 64-bit values, tensor by tensor, from the definition
# ---------------------------------------------------------------------------------------------------------------
def _f32(x):
    return torch.tensor(x, dtype=torch.float32).double().item()


def _hash32(position, seed, step):
    key = (seed + step * 0x9E3779B97F4A7C15) % 2**64
    for shift, factor in ((30, 0xBF58476D1CE4E5B9), (27, 0x94D049BB133111EB), (31, 1)):
        key = ((key ^ (key >> shift)) * factor) % 2**64
    k0, k1 = key % 2**32, key // 2**32

    def fold(x, factor):  # upper and lower half of a 64-bit product, from 16-bit pieces
        low, high = (x % 65536) * factor, (x // 65536) * factor
        mid = high % 65536 * 65536 + low
        return torch.bitwise_xor(mid % 2**32, (high // 65536 + mid // 2**32) % 2**32)

    x = fold(torch.bitwise_xor(position % 2**32, torch.full_like(position, k0)), 0xAC4C1B51)
    x = torch.bitwise_xor(x, torch.bitwise_xor((position // 2**32) * 0x85EBCA6B % 2**32, torch.full_like(position, k1)))
    return fold(x, 0xD6E8FEB5)


def _exact_8_bits(x, chance, positive):
    """x: one tensor's elements. Returns the e4m3 values and the scales, block by block."""
    n = x.numel()
    full = torch.zeros(-(-n // BLOCK) * BLOCK, dtype=torch.float64, device=x.device)
    full[:n] = x
    top = torch.maximum(full.view(-1, BLOCK).abs().max(dim=1).values, torch.tensor(2.0**-100, dtype=torch.float64, device=x.device))
    y = x.abs() * (448.0 / top).repeat_interleave(BLOCK)[:n]
    exponent = torch.floor(torch.log2(torch.clamp(y, min=1e-300)))
    exponent = torch.where(torch.exp2(exponent) > y, exponent - 1, exponent)
    exponent = torch.where(torch.exp2(exponent + 1) <= y, exponent + 1, exponent)
    quantum = torch.exp2(torch.clamp(exponent, min=-6) - 3)
    whole = torch.floor(y / quantum)
    whole = whole + (y / quantum - whole + chance / 65536 >= 1)
    value = torch.clamp(whole * quantum, max=448.0)
    if positive:
        value = torch.where((value == 0) & (x > 0), torch.full_like(value, 2.0**-9), value)
    return torch.where(x < 0, -value, value), top / 448


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    sizes, starts, total = _layout(case)
    lam = [b / sum(s["batches"]) for b in s["batches"]]
    parts = []
    for n, at in zip(sizes, starts):
        g = torch.zeros(n, dtype=torch.float64, device="cuda")
        for k in range(case["K"]):
            g += lam[k] * s["grads"][k, at:at + n].double()
        parts.append(g)
    norm = math.sqrt(sum(float((g * g).sum()) for g in parts))
    if case["op"] == "norm":
        return {"norm": torch.tensor([norm], dtype=torch.float64)}
    factor = min(1.0, case["max_norm"] / norm) if case["max_norm"] > 0 else 1.0
    lr, beta1, beta2, eps, t = _f32(LR), _f32(BETA1), _f32(case["beta2"]), _f32(EPS), case["step"]
    zeros = lambda n: torch.zeros(n, dtype=torch.float64, device="cuda")  # noqa: E731
    out = {"params": zeros(total), "first": zeros(total), "second": zeros(total)}
    if case["state"] == 8:
        out.update(first_scale=zeros(total // BLOCK), second_scale=zeros(total // BLOCK))
    for shape, n, at, g in zip(shapes(case), sizes, starts, parts):
        h = factor * g
        b0, b1 = at // BLOCK, at // BLOCK + -(-n // BLOCK)
        m, u = s["first"][at:at + n].double(), s["second"][at:at + n].double()
        if case["state"] == 8:
            m = m * s["first_scale"][b0:b1].double().repeat_interleave(BLOCK)[:n]
            u = u * s["second_scale"][b0:b1].double().repeat_interleave(BLOCK)[:n]
        m = beta1 * m + (1 - beta1) * h
        u = beta2 * u + (1 - beta2) * h * h
        decay = _f32(DECAY) if len(shape) > 1 else 0.0
        p = s["params"][at:at + n].double() * (1 - lr * decay)
        out["params"][at:at + n] = p - lr * (m / (1 - beta1**t)) / (torch.sqrt(u / (1 - beta2**t)) + eps)
        if case["state"] == 32:
            out["first"][at:at + n], out["second"][at:at + n] = m, u
        else:
            r = _hash32(torch.arange(at, at + n, device="cuda"), s["seed"], t)
            for name, x, chance in (("first", m, r % 65536), ("second", u, r // 65536)):
                value, scale = _exact_8_bits(x, chance.double(), name == "second")
                out[name][at:at + n], out[name + "_scale"][b0:b1] = value, scale
    if case["copy"]:
        out["working"] = out["params"].to(torch.bfloat16).double()
    if case["max_norm"] > 0:
        out["norm"] = torch.tensor([norm], dtype=torch.float64)
    return out
