"""The global norm and the clipping factor in every way in which they are formed: partial sums that the step adds itself (up
to 512), a norm kernel whose last CTA adds them (up to eight for each SM), one fold kernel behind it, two of them (more than
8192 partials); with the aggregate left for the step and with the gradients read again.

A record of the norm kernel is 2048 elements times 4, 2, 1, 1 for 1, 2, 4, 8 fp32 workers (times 8, 4, 2, 1 for bf16 ones), its
partials are two, and every tensor begins a record of its own; the sizes below follow from that and from 148 SMs."""
import math

import numpy as np
import pytest
import torch

import adamw_reference as ref
from helpers import host_grad
from paper_2305_12213_b200 import binding
from test_gpu_adamw import Problem, batches, check_step

pytestmark = pytest.mark.gpu
DEV = "cuda"
LR, B1, B2, EPS = 3e-3, 0.9, 0.95, 1e-8


def aggregate32(grads, b):
    """The aggregate bit for bit: fp32 products of the workers that have samples, added in order within groups of four, the
    groups' sums in order."""
    act = [(np.float32(n / sum(b)), ref.widen(g).astype(np.float32)) for g, n in zip(grads, b) if n > 0]
    total = None
    for i in range(0, len(act), 4):
        group = None
        for w, g in act[i:i + 4]:
            x = w * g
            group = x if group is None else group + x
        total = group if total is None else total + group
    assert total.dtype == np.float32
    return total


def exact_norm(tensors, b):
    return math.sqrt(sum(float(np.sum(np.square(aggregate32(g, b).astype(np.float64)))) for g in tensors))


def is_norm(got, want, n):
    """One rounding to fp32; an fp64 sum of n squares in another order is off by n 2^-53 of itself at most, its root by half of it."""
    return abs(got - want) <= want * (ref.EPS32 + (n + 4) * 2.0**-53)


MODES = [
    # K, sizes: 2 to 8 partials; 684 and 612; 1466 and 1344; 8302 and 8400
    (4, [5000]), (1, [5000, 0, 300]),
    (4, [700_001]), (1, [2_500_000]),
    (4, [1_500_000]), (1, [5_500_003]),
    (4, [8_500_000]), (1, [1000] * 4200),
]


@pytest.mark.parametrize("state8", [False, True])
@pytest.mark.parametrize("K,sizes", MODES)
def test_the_factor_of_every_fold(K, sizes, state8):
    """K = 4 fp32 workers: the aggregate is staged; one: its gradient is read twice.  Three steps of one plan with different
    bounds, the last one above the norm, so that a factor left from the step before shows."""
    prob = Problem(sizes, K, torch.float32, state8, 200 + K, copy=True, fresh=False)
    b, n = batches(K), sum(sizes)
    grads = prob.host_grads()
    norm = ref.norm(grads, b)
    # what the fp32 aggregate's own roundings may move the norm by: the norm of their bounds
    moved = math.sqrt(sum(float(np.sum(np.square(ref.aggregate(g, b)[1]))) for g in grads)) / norm
    # and one rounding of the factor; the bound is an fp32 number
    factor_off = moved + 1.01 * ref.EPS32 + (n + 4) * 2.0**-53
    plan, out = prob.plan(clip=True), torch.zeros(1, device=DEV)
    for t, (share, log) in enumerate([(0.37, True), (0.11, False), (2.0, True)], start=12):
        before, limit = prob.state(), ref.f32(share * norm)
        out.fill_(-1.0)
        plan.step(b, LR, B1, B2, EPS, t, max_norm=limit, seed=8, grad_norm=out if log else None)
        torch.cuda.synchronize()
        assert is_norm(out.item(), exact_norm(grads, b), n) if log else out.item() == -1.0
        check_step(prob, before, grads, b, LR, B1, B2, EPS, t, min(1.0, limit / norm), factor_off if share < 1 else 0.0, seed=8)


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("K", [1, 2, 3, 5, 8, 9, 17, 64])
@pytest.mark.parametrize("shift", [0, 1])
def test_the_norm_is_the_aggregates_to_one_rounding(shift, K, grad):
    """Alone, by a step that does not clip and by one that does, on few and on many partials."""
    for sizes in ([1, 0, 255, 256, 2049, 70_001], [1_300_000, 7]):
        for state8 in (False, True):
            prob = Problem(sizes, K, grad, state8, 300 + K, grad_shift=shift)
            b, out = batches(K), torch.zeros(3, device=DEV)
            want = exact_norm(prob.host_grads(), b)
            binding.GradNormPlan(prob.grads).run(b, out[:1])
            plan = prob.plan(clip=True)
            plan.step(b, LR, B1, B2, EPS, 1, grad_norm=out[1:2])
            plan.step(b, LR, B1, B2, EPS, 2, max_norm=0.5 * want, grad_norm=out[2:])
            for got in out.tolist():
                assert is_norm(got, want, sum(sizes))


def test_aggregate32_against_fp64():
    """The order above is within the bound that the fp64 reference gives any order of so few roundings."""
    prob = Problem([5000], 17, torch.bfloat16, False, 5)
    b = batches(17)
    grads = [host_grad(g[0]) for g in prob.grads]
    want, off = ref.aggregate(grads, b)
    assert np.all(np.abs(aggregate32(grads, b) - want) <= off)
