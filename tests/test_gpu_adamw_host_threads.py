"""Two host threads on one plan and one stream: every call's launches stay together, so each gets its own workers' norm
and a step its own factor."""
import math
import threading

import numpy as np
import pytest
import torch

from paper_2305_12213_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda"
CALLS = 400


def _together(*bodies):
    """The bodies at once; the first exception of any of them."""
    start, errors = threading.Barrier(len(bodies)), []

    def run(body):
        try:
            start.wait(30)
            for i in range(CALLS):
                body(i)
        except BaseException as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=run, args=(body,)) for body in bodies]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    if errors:
        raise errors[0]


def _problem(n, K):
    """Workers of the first half have gradients of 1, the others of 2: any mean over one half is exactly 1 or 2, and its norm
    sqrt(n) or 2 sqrt(n), which fp64 holds to 2^-53 for sums of ones and fours."""
    grads = [[torch.full((n,), 1.0 if k < K // 2 else 2.0, device=DEV)] for k in range(K)]
    first = [1] * (K // 2) + [0] * (K // 2)
    return grads, first, first[::-1], [float(np.float32(v * math.sqrt(n))) for v in (1, 2)]


# few partials, which the step adds; a norm kernel that folds in its last CTA; a fold kernel in between; K = 8: four active
# workers, whose aggregate the norm kernel leaves for the step
@pytest.mark.parametrize("state8", [False, True])
@pytest.mark.parametrize("K", [2, 8])
@pytest.mark.parametrize("n", [5_000, 1_100_000, 6_000_000])
def test_clipped_steps_of_two_threads(n, K, state8):
    grads, b_one, b_two, want = _problem(n, K)
    p = torch.zeros(n, device=DEV)
    dt = torch.float8_e4m3fn if state8 else torch.float32
    m, u = (torch.zeros(n, device=DEV).to(dt) for _ in range(2))
    scales = [[torch.zeros(binding.adamw_scale_elems(n), device=DEV)] for _ in range(2)] if state8 else [None, None]
    plan = binding.AdamWPlan(grads, [p], [m], [u], *scales, clip=True)
    outs = [[torch.zeros(1, device=DEV) for _ in range(CALLS)] for _ in range(2)]
    limit = 0.5 * math.sqrt(n)

    def body(b, out):
        # beta1 = 0: the first moment is factor times gradient, 0.5 whichever half the call averages
        return lambda i: plan.step(b, 0.0, 0.0, 0.9, 1e-8, 1, max_norm=limit, grad_norm=out[i])

    _together(body(b_one, outs[0]), body(b_two, outs[1]))
    for out, w in zip(outs, want):
        assert int((torch.cat(out) != w).sum()) == 0
    got = m.float() * (torch.repeat_interleave(scales[0][0], 256)[:n] if state8 else 1.0)
    # two roundings: limit and factor to fp32 (every product is by 1 or 2); 8 bits: the scale's constant, its product, and
    # code (448, the maximum's) times scale
    assert ((got.double() - 0.5).abs() <= 0.5 * (5 if state8 else 2) * 2.0**-24 * 1.01).all()


@pytest.mark.parametrize("n", [1_100_000, 6_000_000])
def test_norms_of_two_threads(n):
    grads, b_one, b_two, want = _problem(n, 2)
    plan = binding.GradNormPlan(grads)
    outs = [[torch.zeros(1, device=DEV) for _ in range(CALLS)] for _ in range(2)]
    _together(lambda i: plan.run(b_one, outs[0][i]), lambda i: plan.run(b_two, outs[1][i]))
    for out, w in zip(outs, want):
        assert int((torch.cat(out) != w).sum()) == 0
