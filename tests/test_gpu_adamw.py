"""db_aggregate_adamw_multi and db_grad_norm_multi against the fp64 reference, with bounds derived from the number of
fp32 roundings (tests/adamw_reference.py)."""
import math

import numpy as np
import pytest
import torch

import adamw_reference as ref
from helpers import f64, host_grad
from paper_2305_12213_b200 import binding, inputs

pytestmark = pytest.mark.gpu
DEV = "cuda"
E4M3 = torch.float8_e4m3fn
LR, B1, B2, EPS = 3e-3, 0.9, 0.95, 1e-8
SIZES = [1, 0, 255, 256, 257, 2047, 2048, 2049, 31, 5000, 70001]


def place(values, dtype, shift, guard=16):
    """`values` on the GPU, `shift` elements behind an aligned address, with sentinels on both sides."""
    n = values.numel()
    back = torch.full((n + 2 * guard + shift,), 7.0, device=DEV).to(dtype)
    back[guard + shift:guard + shift + n] = values.to(DEV).to(dtype)
    view = back[guard + shift:guard + shift + n]
    view.back = back
    return view


def untouched(view, guard=16):
    n, off = view.numel(), view.storage_offset()
    back = view.back.float()
    return bool((back[:off] == 7).all() and (back[off + n:] == 7).all())


class Problem:
    def __init__(self, sizes, K, grad, state8, seed, copy=False, shift=0, grad_shift=0, fresh=True, std=1e-2):
        rng = np.random.default_rng(seed)
        self.sizes, self.K, self.state8 = sizes, K, state8
        self.wd = [0.1 if t % 2 else 0.0 for t in range(len(sizes))]
        draw = lambda n, s: torch.tensor(rng.standard_normal(n) * s, dtype=torch.float32)  # noqa: E731
        self.grads = [[place(draw(n, std * 10.0 ** rng.uniform(-2, 1)), grad, grad_shift) for n in sizes] for _ in range(K)]
        self.p = [place(draw(n, 0.02), torch.float32, shift) for n in sizes]
        self.copy = [place(torch.zeros(n), torch.bfloat16, shift) for n in sizes] if copy else None
        dt = E4M3 if state8 else torch.float32
        zero = lambda n: torch.zeros(n)  # noqa: E731
        blocks = [binding.adamw_scale_elems(n) for n in sizes]
        if fresh:
            self.m, self.u = ([place(zero(n), dt, shift) for n in sizes] for _ in range(2))
            self.ms, self.us = ([place(zero(n), torch.float32, 0) for n in blocks] for _ in range(2))
        elif state8:
            self.m = [place(draw(n, 100).clamp(-448, 448), dt, shift) for n in sizes]
            self.u = [place((draw(n, 60).abs() + 1).clamp(0, 448), dt, shift) for n in sizes]
            self.ms = [place(draw(n, 1e-5).abs() + 1e-6, torch.float32, 0) for n in blocks]
            self.us = [place(draw(n, 1e-7).abs() + 1e-8, torch.float32, 0) for n in blocks]
        else:
            self.m = [place(draw(n, 1e-3), dt, shift) for n in sizes]
            self.u = [place(draw(n, 1e-2).square(), dt, shift) for n in sizes]
        if not state8:
            self.ms = self.us = None

    def plan(self, clip=False):
        return binding.AdamWPlan(self.grads, self.p, self.m, self.u, self.ms, self.us, self.copy, self.wd, clip)

    def clone(self):
        c = object.__new__(Problem)
        c.__dict__.update(self.__dict__)
        for name in ("p", "m", "u", "ms", "us", "copy"):
            old = getattr(self, name)
            new = None
            if old is not None:
                new = []
                for x in old:
                    back = x.back.clone()
                    v = back[x.storage_offset():x.storage_offset() + x.numel()]
                    v.back = back
                    new.append(v)
            setattr(c, name, new)
        return c

    def state(self):
        """fp64 (p, m, u) of every tensor as the kernel sees them, and a code's own values."""
        def wide(x, s):
            if not self.state8:
                return f64(x)
            v = ref.e4m3_values(x.view(torch.uint8).cpu().numpy())
            return (v.astype(np.float32) * np.repeat(s.cpu().numpy(), ref.BLOCK)[:v.size]).astype(np.float64)
        ms, us = self.ms or [None] * len(self.sizes), self.us or [None] * len(self.sizes)
        return [(f64(p), wide(m, s), wide(u, r)) for p, m, u, s, r in zip(self.p, self.m, self.u, ms, us)]

    def host_grads(self):
        return [[host_grad(g[t]) for g in self.grads] for t in range(len(self.sizes))]

    def all_tensors(self):
        return [x for part in (self.p, self.m, self.u, self.ms or [], self.us or [], self.copy or []) for x in part]


def check_step(prob, before, grads, b, lr, b1, b2, eps, t, factor=1.0, factor_off=0.0, seed=0):
    """The state after one step from `before`, tensor by tensor, within the bounds."""
    position = 0
    for i, n in enumerate(prob.sizes):
        (p, m, u), (po, mo, uo) = ref.step(grads[i], b, *before[i], lr, b1, b2, eps, t, prob.wd[i], factor, factor_off)
        assert np.all(np.abs(f64(prob.p[i]) - p) <= po), f"params of tensor {i}, step {t}"
        if not prob.state8:
            assert np.all(np.abs(f64(prob.m[i]) - m) <= mo), f"first moment of tensor {i}, step {t}"
            assert np.all(np.abs(f64(prob.u[i]) - u) <= uo), f"second moment of tensor {i}, step {t}"
        else:
            for name, codes, scales, x, off, second in (("first", prob.m[i], prob.ms[i], m, mo, False),
                                                        ("second", prob.u[i], prob.us[i], u, uo, True)):
                if n == 0:
                    continue
                lo, hi, s, s_off = ref.code_range(x, off, position, seed, t, second)
                got = ref.e4m3_values(codes.view(torch.uint8).cpu().numpy())
                assert np.all((np.abs(got) >= lo) & (np.abs(got) <= hi)), f"{name} codes of tensor {i}, step {t}"
                sure = np.abs(x) > off
                assert np.all((got[sure] == 0) | ((got[sure] > 0) == (x[sure] > 0)))
                assert np.all(np.abs(f64(scales) - s) <= s_off), f"{name} scales of tensor {i}, step {t}"
        if prob.copy is not None:
            assert torch.equal(prob.copy[i], prob.p[i].to(torch.bfloat16))
        position += -(-n // ref.BLOCK) * ref.BLOCK
    assert all(untouched(x) for x in prob.all_tensors())


def batches(K):
    return [3 + 5 * k % 17 for k in range(K)]


@pytest.mark.parametrize("state8", [False, True])
@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("K", [1, 2, 3, 5, 8, 9, 17, 64])
def test_steps_from_zero(K, grad, state8):
    prob = Problem(SIZES, K, grad, state8, 10 + K, copy=K % 2 == 1)
    plan, b = prob.plan(), batches(K)
    for t in range(1, 4):
        before, grads = prob.state(), prob.host_grads()
        plan.step(b, LR, B1, B2, EPS, t, seed=99)
        torch.cuda.synchronize()
        check_step(prob, before, grads, b, LR, B1, B2, EPS, t, seed=99)
    plan.close()


@pytest.mark.parametrize("state8", [False, True])
@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift,grad_shift", [(0, 1), (1, 0), (3, 2), (4, 4), (8, 8)])
def test_any_alignment_gives_the_same_bits(shift, grad_shift, grad, state8):
    a = Problem(SIZES, 3, grad, state8, 5, copy=True, fresh=False)
    c = Problem(SIZES, 3, grad, state8, 5, copy=True, fresh=False, shift=shift, grad_shift=grad_shift)
    b, n = [4, 1, 9], torch.zeros(2, device=DEV)
    before, grads = c.state(), c.host_grads()
    for prob, out, clip in ((a, n[:1], False), (c, n[1:], False)):
        prob.plan(clip).step(b, LR, B1, B2, EPS, 30, seed=2**63 + 1, grad_norm=out)
    torch.cuda.synchronize()
    check_step(c, before, grads, b, LR, B1, B2, EPS, 30, seed=2**63 + 1)
    for x, y in zip(a.all_tensors(), c.all_tensors()):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)) if x.dtype == E4M3 else torch.equal(x, y)
    assert abs(n[0].item() - n[1].item()) <= 2 * ref.EPS32 * n[0].item()     # other lanes, other fp32 partial sums of eight


@pytest.mark.parametrize("state8", [False, True])
@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("K", [1, 2, 3, 5, 8, 13, 40])
def test_every_worker_at_its_own_offset(K, grad, state8):
    """Worker k's gradients lie k % 9 elements behind an aligned address, between NaNs: the same bits as with all of them
    aligned, for whole and for shorter blocks."""
    sizes = SIZES + [7001]
    a = Problem(sizes, K, grad, state8, 44, copy=True, fresh=False)
    c = a.clone()
    c.grads = []
    for k, rows in enumerate(a.grads):
        at = 16 + (k + 1) % 9                                        # K = 1: an odd element
        backs = [torch.full((x.numel() + 48,), math.nan, dtype=grad, device=DEV) for x in rows]
        c.grads.append([back[at:at + x.numel()].copy_(x) for back, x in zip(backs, rows)])
    b, n = batches(K), torch.zeros(2, device=DEV)
    for prob, out in ((a, n[:1]), (c, n[1:])):
        plan = prob.plan(clip=True)
        plan.step(b, LR, B1, B2, EPS, 3, seed=8)
        plan.step(b, LR, B1, B2, EPS, 4, max_norm=1e9, seed=8, grad_norm=out)
    torch.cuda.synchronize()
    assert n[0].item() > 0 and abs(n[0].item() - n[1].item()) <= 2 * ref.EPS32 * n[0].item()     # other lanes' fp32 squares
    for x, y in zip(a.all_tensors(), c.all_tensors()):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)) if x.dtype == E4M3 else torch.equal(x, y)
    assert all(untouched(x) for x in c.all_tensors())


def norm_tolerance(K):
    """Relative bound of the fp32 norm: the aggregate's K roundings act on single elements (at most K 2^-24 (sum of
    magnitudes / magnitude), here about sqrt(K) larger at most), a lane's eight squares 8 2^-24 / 2, the result 2^-24."""
    return (4 * K + 6) * ref.EPS32


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("K", [1, 2, 4, 7, 16])
@pytest.mark.parametrize("state8", [False, True])
def test_clipped_steps(state8, K, grad):
    """K = 1, 2 reads the gradients twice, the others stage the aggregate; also with every other tensor unaligned."""
    for grad_shift, shift in ((0, 0), (1, 0), (0, 1)):
        prob = Problem(SIZES, K, grad, state8, 60 + K, copy=True, shift=shift, grad_shift=grad_shift, fresh=False)
        b, out = batches(K), torch.zeros(1, device=DEV)
        before, grads = prob.state(), prob.host_grads()
        norm = ref.norm(grads, b)
        limit = ref.f32(0.37 * norm)
        plan = prob.plan(clip=True)
        plan.step(b, LR, B1, B2, EPS, 12, max_norm=limit, seed=8, grad_norm=out)
        torch.cuda.synchronize()
        assert abs(out.item() - norm) <= norm_tolerance(K) * norm
        check_step(prob, before, grads, b, LR, B1, B2, EPS, 12, limit / norm, norm_tolerance(K) + 2 * ref.EPS32, seed=8)


def test_a_bound_above_the_norm_changes_nothing():
    for K in (2, 6):
        a = Problem(SIZES, K, torch.float32, True, 31, fresh=False)
        c = a.clone()
        b = batches(K)
        a.plan().step(b, LR, B1, B2, EPS, 4, seed=3)
        c.plan(clip=True).step(b, LR, B1, B2, EPS, 4, max_norm=1e9, seed=3)
        torch.cuda.synchronize()
        for x, y in zip(a.all_tensors(), c.all_tensors()):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("K,sizes", [(1, [1]), (1, SIZES), (3, [256]), (4, SIZES), (8, [3_000_017]), (20, [5000, 0, 70001]),
                                     (2, [37] * 3000)])
def test_norm(K, sizes, grad):
    for shift in (0, 1):
        prob = Problem(sizes, K, grad, False, 77, grad_shift=shift)
        b, out = batches(K), torch.full((3,), 5.0, device=DEV)
        plan = binding.GradNormPlan(prob.grads)
        want = ref.norm(prob.host_grads(), b)
        plan.run(b, out[1:2])
        torch.cuda.synchronize()
        assert out[0].item() == out[2].item() == 5.0
        assert abs(out[1].item() - want) <= norm_tolerance(K) * want
        first = out[1].item()
        plan.run(b, out[1:2])
        assert out[1].item() == first                                        # the sum's order is fixed
        step = torch.zeros(1, device=DEV)
        prob.plan().step(b, 0.0, B1, B2, EPS, 1, grad_norm=step)              # as the by-product of a step that does not clip
        assert abs(step.item() - want) <= norm_tolerance(K) * want


def test_norm_of_very_large_and_very_small_gradients():
    for size in (1e25, 3e30, 1e-25, 1e-40, 0.0):
        g = torch.full((3000,), size, device=DEV)
        g[5] = 0.0
        out = torch.ones(1, device=DEV)
        binding.GradNormPlan([[g]]).run([4], out)
        want = float(np.float32(size)) * math.sqrt(2999)
        assert abs(out.item() - want) <= norm_tolerance(1) * want + 2.0**-149
    # one large element among ordinary ones, and a mixture of large and vanishing ones in one lane
    g = torch.full((3000,), 1e-3, device=DEV)
    g[100:103] = torch.tensor([1e20, 1e-30, 2e20], device=DEV)
    out = torch.ones(1, device=DEV)
    binding.GradNormPlan([[g]]).run([4], out)
    want = float(f64(g).__pow__(2).sum() ** 0.5)
    assert abs(out.item() - want) <= norm_tolerance(1) * want


def test_two_stage_fold_of_a_step_with_norm():
    n = 2048 * 8192 + 2048 * 5 + 3                                           # more tiles than one fold stage takes
    g = inputs.normal(n, 1e-3, 1, DEV)
    p, m, u = (torch.zeros(n, device=DEV) for _ in range(3))
    out = torch.zeros(1, device=DEV)
    binding.AdamWPlan([[g]], [p], [m], [u]).step([1], 1e-3, B1, B2, EPS, 1, grad_norm=out)
    want = g.double().square().sum().sqrt().item()
    assert abs(out.item() - want) <= norm_tolerance(1) * want


@pytest.mark.parametrize("state8", [False, True])
def test_worker_without_samples_is_never_read(state8):
    a = Problem(SIZES, 4, torch.float32, state8, 9, fresh=False)
    for g in a.grads[1] + a.grads[3]:
        g.fill_(float("nan"))
    b, out = [4, 0, 7, 0], torch.zeros(1, device=DEV)
    before = a.state()
    grads = a.host_grads()
    a.plan(clip=True).step(b, LR, B1, B2, EPS, 3, max_norm=1e9, seed=1, grad_norm=out)
    torch.cuda.synchronize()
    check_step(a, before, grads, b, LR, B1, B2, EPS, 3, seed=1)
    assert math.isfinite(out.item())


def test_nan_and_infinity_stay_in_their_element_or_block():
    """32-bit states: the element alone.  8 bits: its block of 256 loses its moments, no other block does."""
    for state8 in (False, True):
        for bad in (float("nan"), float("inf")):
            a = Problem([1000, 300], 2, torch.float32, state8, 4, fresh=False)
            clean = a.clone()
            clean.plan().step([1, 2], LR, B1, B2, EPS, 5, seed=6)
            torch.cuda.synchronize()
            kept = a.grads[0][0][300].item()
            a.grads[0][0][300] = bad
            a.plan().step([1, 2], LR, B1, B2, EPS, 5, seed=6)
            torch.cuda.synchronize()
            a.grads[0][0][300] = kept
            others = torch.arange(1000, device=DEV) != 300
            assert torch.equal(a.p[0][others], clean.p[0][others]) and torch.equal(a.p[1], clean.p[1])
            assert not math.isfinite(a.p[0][300].item())
            if state8:
                assert torch.isnan(a.ms[0][1]) and torch.isnan(a.us[0][1])
                for s, c in ((a.ms, clean.ms), (a.us, clean.us)):
                    assert torch.equal(s[0][[0, 2, 3]], c[0][[0, 2, 3]]) and torch.equal(s[1], c[1])
                for x, y in ((a.m, clean.m), (a.u, clean.u)):
                    got, want = x[0].view(torch.uint8), y[0].view(torch.uint8)
                    assert (got[256:512] == 0).all() and torch.equal(got[512:], want[512:]) and torch.equal(got[:256], want[:256])
            else:
                assert torch.equal(a.m[0][others], clean.m[0][others]) and torch.equal(a.u[0][others], clean.u[0][others])


def test_clipping_with_a_norm_that_is_not_finite():
    """NaN: no clipping, the NaN stays in its element.  Infinity: the factor is 0, so finite elements see a zero gradient."""
    for bad in (float("nan"), float("inf")):
        a = Problem([1000], 1, torch.float32, False, 4, fresh=False)
        c = a.clone()
        c.grads = [[g.clone() if bad != bad else torch.zeros_like(g) for g in a.grads[0]]]
        c.plan().step([1], LR, B1, B2, EPS, 5)
        torch.cuda.synchronize()
        a.grads[0][0][7] = bad
        out = torch.zeros(1, device=DEV)
        a.plan(clip=True).step([1], LR, B1, B2, EPS, 5, max_norm=1e-3, grad_norm=out)
        torch.cuda.synchronize()
        others = torch.arange(1000, device=DEV) != 7
        assert not math.isfinite(out.item()) and math.isnan(a.p[0][7].item())
        for x, y in ((a.p, c.p), (a.m, c.m), (a.u, c.u)):
            assert torch.equal(x[0][others], y[0][others])


def test_blocks_of_zeros_of_tiny_and_of_large_values():
    """Moments of 0, around the smallest scale 2^-100 / 448, and of 1e18; a second moment > 0 is never held as 0."""
    for size in (0.0, 1e-30, 1e-15, 1e18):
        a = Problem([600], 1, torch.float32, True, 4, std=0.0)
        a.grads[0][0].copy_(inputs.normal(600, 1.0, 3, DEV) * size)
        for t in range(1, 4):
            before, grads = a.state(), a.host_grads()
            a.plan().step([1], LR, B1, B2, EPS, t, seed=4)
            torch.cuda.synchronize()
            check_step(a, before, grads, [1], LR, B1, B2, EPS, t, seed=4)
            if size >= 1e-15:
                assert (a.u[0].view(torch.uint8)[a.grads[0][0] != 0] != 0).all()
    a = Problem([256], 1, torch.float32, True, 4, std=0.0)
    a.grads[0][0].fill_(1e-12)
    a.grads[0][0][9] = 1e6                                                   # 36 decades of squares in one block
    a.plan().step([1], LR, B1, B2, EPS, 1, seed=4)
    torch.cuda.synchronize()
    codes = a.u[0].view(torch.uint8)
    assert codes[9].item() == 0x7E and (codes[:9] == 1).all() and (codes[10:] == 1).all()


def test_rounding_follows_a_slow_average():
    """beta2 = 0.999 moves u by a thousandth a step, far below an 8-bit step.  After 800 steps on a constant g^2 the
    mean of u over 40,000 elements is what fp64 gives: every step's rounding is unbiased given the state before it, so
    the error of the mean is a martingale; a rounding's standard deviation is at most q / 2 with q <= u / 8, and a step
    that moves u by d is rounded with variance at most d q, where d <= 2e-3 u (decay and scale drift).  Summed over
    the 1000 steps that the average remembers and divided by sqrt(40,000): sqrt(500 * 2e-3 / 8) / 200 = 0.0018;
    five of those are 0.009.  Elements never sit at the block's maximum alone, where nothing is rounded."""
    n = 40_000
    g = torch.ones(n, device=DEV)
    g[::256] = 4.0                                                            # one larger element in each block sets its scale
    p, m, u = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV).to(E4M3), torch.zeros(n, device=DEV).to(E4M3)
    ms, us = (torch.zeros(binding.adamw_scale_elems(n), device=DEV) for _ in range(2))
    plan = binding.AdamWPlan([[g]], [p], [m], [u], [ms], [us])
    # a start off the average, so that it has somewhere to go
    u.view(torch.uint8).fill_(0x50)
    us.fill_(0.002)
    start = float(ref.e4m3_values(np.array([0x50], np.uint8))[0]) * 0.002
    for t in range(1, 801):
        plan.step([1], 0.0, B1, 0.999, EPS, t, seed=17)
    torch.cuda.synchronize()
    keep = ref.f32(0.999) ** 800
    ones = torch.arange(n, device=DEV) % 256 != 0
    got = (u.float() * torch.repeat_interleave(us, 256)[:n])[ones].mean().item()
    want = keep * start + (1 - keep)
    assert abs(got - want) <= 0.009 * want
    got = (m.float() * torch.repeat_interleave(ms, 256)[:n])[ones].mean().item()
    assert abs(got - 1.0) <= 0.009


def test_capture_and_replay():
    for state8, max_norm in ((False, 0.0), (True, 0.5)):
        a = Problem(SIZES, 3, torch.bfloat16, state8, 6, copy=True, fresh=False)
        c = a.clone()
        b, out = [1, 2, 3], torch.zeros(1, device=DEV)
        plan, other = a.plan(clip=True), c.plan(clip=True)
        for _ in range(3):
            other.step(b, LR, B1, B2, EPS, 9, max_norm=max_norm, seed=5)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            plan.step(b, LR, B1, B2, EPS, 9, max_norm=max_norm, seed=5, grad_norm=out)
        for _ in range(3):
            graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(a.all_tensors(), c.all_tensors()):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)) if x.dtype == E4M3 else torch.equal(x, y)
        assert out.item() > 0


def test_steps_back_to_back_see_each_other():
    """Kernels may be scheduled before their predecessor has ended: 20 steps without a wait are 20 steps with one."""
    for state8 in (False, True):
        a = Problem([300_000, 5000], 5, torch.bfloat16, state8, 8, copy=True)
        c = a.clone()
        pa, pc, b = a.plan(clip=True), c.plan(clip=True), batches(5)
        for t in range(1, 21):
            limit = 0.5 if t % 2 else 0.0
            pa.step(b, LR, B1, B2, EPS, t, max_norm=limit, seed=t)
        for t in range(1, 21):
            limit = 0.5 if t % 2 else 0.0
            pc.step(b, LR, B1, B2, EPS, t, max_norm=limit, seed=t)
            torch.cuda.synchronize()
        torch.cuda.synchronize()
        for x, y in zip(a.all_tensors(), c.all_tensors()):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)) if x.dtype == E4M3 else torch.equal(x, y)


def test_other_streams():
    a = Problem([100_000], 2, torch.float32, False, 8)
    c = a.clone()
    b = [1, 2]
    plan, s = a.plan(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    plan.step(b, LR, B1, B2, EPS, 1, stream=s)
    with torch.cuda.stream(s):
        plan.step(b, LR, B1, B2, EPS, 2)
    torch.cuda.current_stream().wait_stream(s)
    other = c.plan()
    other.step(b, LR, B1, B2, EPS, 1)
    other.step(b, LR, B1, B2, EPS, 2)
    torch.cuda.synchronize()
    assert torch.equal(a.p[0], c.p[0]) and torch.equal(a.m[0], c.m[0])


def test_more_elements_than_32_bits_count():
    """8-bit moments, bf16 gradient, 2^32 + 777 elements of one tensor: the end of it and both sides of 2^32 and 2^31."""
    n = 2**32 + 777
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    p, g = torch.zeros(n, device=DEV), torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    m, u = (torch.zeros(n, dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2))
    ms, us = (torch.zeros(binding.adamw_scale_elems(n), device=DEV) for _ in range(2))
    spots = [(0, 512), (2**31 - 512, 2**31 + 512), (2**32 - 512, 2**32 + 777)]
    for i, (lo, hi) in enumerate(spots):
        g[lo:hi] = inputs.normal(hi - lo, 1.0, 40 + i, DEV).to(torch.bfloat16)
        p[lo:hi] = inputs.normal(hi - lo, 0.02, 50 + i, DEV)
    before = [(f64(p[lo:hi]), host_grad(g[lo:hi])) for lo, hi in spots]
    out = torch.zeros(1, device=DEV)
    binding.AdamWPlan([[g]], [p], [m], [u], [ms], [us]).step([1], LR, B1, B2, EPS, 1, seed=11, grad_norm=out)
    torch.cuda.synchronize()
    for (lo, hi), (p0, hg) in zip(spots, before):
        zero = np.zeros(hi - lo)
        (pr, mr, ur), (po, mo, uo) = ref.step([hg], [1], p0, zero, zero, LR, B1, B2, EPS, 1)
        assert np.all(np.abs(f64(p[lo:hi]) - pr) <= po)
        for codes, x, off, second in ((m, mr, mo, False), (u, ur, uo, True)):
            a, z, _, _ = ref.code_range(x, off, lo, 11, 1, second)
            got = np.abs(ref.e4m3_values(codes[lo:hi].view(torch.uint8).cpu().numpy()))
            assert np.all((got >= a) & (got <= z))
    assert not p[2**31 + 512:2**31 + 4096].any() and not m.view(torch.uint8)[2**31 + 512:2**31 + 4096].any()
    want = math.sqrt(sum(float((ref.widen(hg) ** 2).sum()) for _, hg in before))
    assert abs(out.item() - want) <= norm_tolerance(1) * want


def test_step_refusals():
    a = Problem([64, 128], 2, torch.float32, False, 3)
    kept = [x.clone() for x in a.all_tensors()]
    plan = a.plan()
    ok = dict(b=[1, 1], lr=LR, beta1=B1, beta2=B2, eps=EPS, step=1)
    nan, inf = float("nan"), float("inf")
    for kw in (dict(b=[0, 0]), dict(b=[1, -1]), dict(lr=nan), dict(lr=inf), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0),
               dict(beta2=nan), dict(eps=-1.0), dict(eps=inf), dict(step=0), dict(max_norm=-1.0), dict(max_norm=nan),
               dict(max_norm=inf), dict(max_norm=1.0)):                       # the last: the plan was made without clipping
        with pytest.raises(binding.DynbatchError) as ei:
            plan.step(**{**ok, **kw})
        assert ei.value.status == binding.DB_ERR_ARG
    with pytest.raises(ValueError):
        plan.step(**{**ok, "b": [1]})
    for bad in (torch.zeros(1, dtype=torch.float64, device=DEV), torch.zeros(1)):
        with pytest.raises((TypeError, ValueError)):
            plan.step(**ok, grad_norm=bad)
    norm = binding.GradNormPlan(a.grads)
    with pytest.raises(binding.DynbatchError):
        norm.run([0, 0], torch.zeros(1, device=DEV))
    with pytest.raises(binding.DynbatchError) as ei:
        norm.run([1, 1], None)
    assert ei.value.status == binding.DB_ERR_NULL
    for kw in (dict(first_moment=a.p), dict(params_bf16=[x.view(torch.bfloat16)[::2] for x in a.m])):
        with pytest.raises((binding.DynbatchError, TypeError)):
            binding.AdamWPlan(**{**dict(grads=a.grads, params=a.p, first_moment=a.m, second_moment=a.u), **kw})
    with pytest.raises(TypeError):
        binding.AdamWPlan(a.grads, a.p, a.m, [x.to(E4M3) for x in a.u])       # moments of two types
    with pytest.raises(binding.DynbatchError):
        binding.AdamWPlan(a.grads, a.p, [x.to(E4M3) for x in a.m], [x.to(E4M3) for x in a.u])      # no scales
    with pytest.raises(ValueError):
        binding.AdamWPlan(a.grads, a.p, a.m, a.u, weight_decay=[0.1])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a.all_tensors(), kept))


def test_plan_is_refused_in_a_capture_and_the_capture_goes_on():
    a = Problem([64], 1, torch.float32, False, 3)
    x = torch.zeros(4, device=DEV)
    torch.cuda.synchronize()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        with pytest.raises(binding.DynbatchError) as ei:
            a.plan()
        assert ei.value.status == binding.DB_ERR_UNSUPPORTED
        x += 1
    graph.replay()
    torch.cuda.synchronize()
    assert x.sum().item() == 4


def test_empty_list_leaves_the_norm():
    z = torch.zeros(0, device=DEV)
    out = torch.full((1,), 3.0, device=DEV)
    binding.AdamWPlan([[z]], [z.clone()], [z.clone()], [z.clone()], clip=True).step([1], LR, B1, B2, EPS, 1, 1.0, 0, out)
    binding.GradNormPlan([[z]]).run([1], out)
    assert out.item() == 3.0


@pytest.mark.parametrize("state8", [False, True])
def test_training_the_classifier_with_workers_clipping_and_adamw(state8):
    """The operators as they are used: ragged worker gradients of the softmax classifier (grouped call), their global
    norm for the log, a clipped AdamW step on the same stream, ten times; each step is checked from the state it
    started from."""
    bs, D, C = [5, 24, 11], 96, 40
    X, y, W = inputs.softmax_problem(bs, D, C, seed=5, device=DEV)
    offs = np.concatenate([[0], np.cumsum(bs)]).tolist()
    G = [torch.empty(D, C, device=DEV) for _ in bs]
    ws = torch.empty(binding.worker_grad_grouped_workspace_bytes(offs[-1], 3, D, C), dtype=torch.uint8, device=DEV)
    prob = Problem([D * C], 3, torch.float32, state8, 1, copy=True)
    prob.p[0].copy_(W.view(-1))
    prob.grads = [[g.view(-1)] for g in G]
    plan, log = prob.plan(clip=True), binding.GradNormPlan(prob.grads)
    seen, inside = torch.zeros(1, device=DEV), torch.zeros(1, device=DEV)
    for t in range(1, 11):
        binding.worker_grad_grouped(X, y, prob.p[0].view(D, C), offs, G, None, ws)
        torch.cuda.synchronize()
        before, grads = prob.state(), prob.host_grads()
        norm = ref.norm(grads, bs)
        limit = ref.f32(0.8 * norm) if t % 2 else ref.f32(2 * norm)
        log.run(bs, seen)
        plan.step(bs, 1e-2, B1, B2, EPS, t, max_norm=limit, seed=t, grad_norm=inside)
        torch.cuda.synchronize()
        assert abs(seen.item() - norm) <= norm_tolerance(3) * norm and abs(inside.item() - norm) <= norm_tolerance(3) * norm
        check_step(prob, before, grads, bs, 1e-2, B1, B2, EPS, t, min(1.0, limit / norm), norm_tolerance(3) + 2 * ref.EPS32, seed=t)
    assert binding.worker_grad_status(ws) == 0


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("K", [1, 3, 8, 13])
def test_codes_are_the_definitions_exactly(K, grad):
    """The same step with 32-bit moments, from the values that the codes stand for, gives the moments before they are
    rounded, bit for bit; from them the definition in fp64 gives every code, with no element left over, and every
    scale is the maximum times fp32's 1/448.  Elements next to a border between two codes, and the block's maximum, are among them:
    two million elements."""
    n = 1_000_003
    a = Problem([n, 1_000_000], K, grad, True, 91, fresh=False)
    wide = object.__new__(Problem)
    wide.__dict__.update(a.__dict__)
    wide.p = [x.clone() for x in a.p]
    vals = a.state()
    wide.m, wide.u = ([torch.tensor(v[i], dtype=torch.float32, device=DEV) for v in vals] for i in (1, 2))
    wide.ms = wide.us = None
    b = batches(K)
    for prob in (a, wide):
        prob.plan(clip=True).step(b, LR, B1, B2, EPS, 6, max_norm=0.5, seed=12)
    torch.cuda.synchronize()
    position = 0
    for t, size in enumerate(a.sizes):
        assert torch.equal(a.p[t], wide.p[t])
        for codes, scales, x, second in ((a.m[t], a.ms[t], f64(wide.m[t]), False), (a.u[t], a.us[t], f64(wide.u[t]), True)):
            top = ref.block_max(x)
            r = ref.random_bits(position + np.arange(size), 12, 6)
            chance = (r >> np.uint64(16) if second else r & np.uint64(0xFFFF)).astype(np.float64)
            want = ref.round_up_by_chance(np.abs(x) * 448 / np.repeat(top, 256)[:size], chance)
            if second:
                want = np.where(x > 0, np.maximum(want, 2.0**-9), want)
            got = ref.e4m3_values(codes.view(torch.uint8).cpu().numpy())
            assert np.array_equal(got, np.where(x < 0, -want, want))
            assert np.array_equal(f64(scales), (top.astype(np.float32) * np.float32(1 / 448)).astype(np.float64))
        position += -(-size // 256) * 256


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("K", [1, 2, 3, 4, 5, 6, 7, 8, 9, 12, 13, 17, 35])
@pytest.mark.parametrize("state8", [False, True])
def test_a_long_run_of_blocks_is_its_pieces(state8, K, grad):
    """A tensor of 10.2M elements, of which every warp takes several blocks in turn, against the same memory as a list of
    tensors of 2048 and 4096 elements, of which it takes one: the same bits, clipped and not, also with gradients at odd
    elements and a last block that is shorter."""
    sizes = [2048, 4096] * 1666 + [2048 + 77]
    n = sum(sizes)
    starts = np.concatenate([[0], np.cumsum(sizes)[:-1]]).tolist()
    g = [torch.empty(n + 1, dtype=grad, device=DEV).normal_(0, 1e-2) for _ in range(K)]
    dt = E4M3 if state8 else torch.float32
    blocks = binding.adamw_scale_elems(n)

    def fresh():
        p = inputs.normal(n, 0.02, 5, DEV)
        m, u = (torch.zeros(n, device=DEV).to(dt) for _ in range(2))
        s = [torch.zeros(blocks, device=DEV) for _ in range(2)] if state8 else None
        return p, torch.zeros(n, dtype=torch.bfloat16, device=DEV), m, u, s

    def cut(t, unit=1):
        return [t[a // unit:a // unit + -(-k // unit)] for a, k in zip(starts, sizes)]

    for shift in (0, 1):
        rows = [x[shift:shift + n] for x in g]
        whole, parts = fresh(), fresh()
        p, w, m, u, s = whole
        one = binding.AdamWPlan([[x] for x in rows], [p], [m], [u], *([[s[0]], [s[1]]] if state8 else [None, None]), [w], clip=True)
        p, w, m, u, s = parts
        many = binding.AdamWPlan([cut(x) for x in rows], cut(p), cut(m), cut(u),
                                 *([cut(s[0], 256), cut(s[1], 256)] if state8 else [None, None]), cut(w), clip=True)
        b, norms = batches(K), torch.zeros(2, device=DEV)
        for t, limit in ((1, 0.0), (2, 1e9), (3, 3.0)):
            one.step(b, LR, B1, B2, EPS, t, limit, 7, norms[:1] if limit else None)
            many.step(b, LR, B1, B2, EPS, t, limit, 7, norms[1:] if limit else None)
        torch.cuda.synchronize()
        # both sums are fp64, so the norms are the same float (but for one pair in 10^8) and the third step's factor, too
        assert norms[0].item() == norms[1].item() > 3.0
        for x, y in zip(whole[:4], parts[:4]):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
        if state8:
            assert torch.equal(whole[4][0], parts[4][0]) and torch.equal(whole[4][1], parts[4][1])


def test_a_plan_that_is_dropped_behind_a_step_on_another_stream():
    """The records' memory is not handed out again while the step's kernels may still read it.  (Addresses are compared;
    nothing is written there.)"""
    n = 1_000_000
    a = Problem([n], 1, torch.float32, False, 8)
    s = torch.cuda.Stream()
    plan = a.plan()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)                      # the step starts some milliseconds later
    plan.step([1], LR, B1, B2, EPS, 1, stream=s)
    begin, size = plan.table.data_ptr(), plan.table.numel()
    plan.close()
    del plan
    others = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(4)]
    assert not s.query()
    assert all(x.data_ptr() + size <= begin or begin + size <= x.data_ptr() for x in others)
    torch.cuda.synchronize()
