"""Every kernel of the layers' products against 64 bits: the bodies and bounds of test_gpu_layers at sizes for which the plan picks
each tile shape, whole and cut (test_layers_plan checks that it does)."""
import pytest
import torch

import layers_cases as cases
import test_gpu_layers as layers
from paper_2305_12213_b200 import binding

pytestmark = pytest.mark.gpu
bf16 = torch.bfloat16


def test_the_plan_of_this_device_reaches_every_kernel():
    got = cases.plans(binding.bench_layer_plan)
    assert len(got) >= 8 * len(cases.SHAPES) * 2 - 2, sorted(got)


@pytest.mark.parametrize("rows,n,m,bias,residual,act,kept,pitch,shift", cases.LINEAR)
def test_linear(rows, n, m, bias, residual, act, kept, pitch, shift):
    layers.test_linear(rows, n, m, bias, residual, act, kept, pitch, shift)


@pytest.mark.parametrize("rows,n,m,residual,act,kept,pitch,shift", cases.FFN)
def test_gated_ffn(rows, n, m, residual, act, kept, pitch, shift):
    layers.test_gated_ffn(rows, n, m, residual, act, kept, pitch, shift)


@pytest.mark.parametrize("rows,n,m", [(3000, 1032, 1544), (100, 1024, 1024), (162, 2799, 2872), (9000, 72, 200)])
def test_wanted_gradients_alone_and_within_the_workspace(rows, n, m):
    """Every choice of gradients has a plan of its own: the same values up to the order of the sums, and room for its pieces."""
    x, dy = layers.normal(1, rows, n), layers.normal(2, rows, n)
    wg, wu, wd = layers.normal(3, n, m, std=n**-0.5), layers.normal(4, n, m, std=n**-0.5), layers.normal(5, m, n, std=m**-0.5)
    keep = {"gate": layers.normal(6, rows, m), "up": layers.normal(7, rows, m)}
    size = binding.gated_ffn_grad_workspace_bytes(rows, n, m)
    room = torch.full((size + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
    ws, behind = room[:size], room[size:]
    like = {"dx": x, "dw_gate": wg, "dw_up": wu, "dw_down": wd}

    def run(names, dtype):
        out = {k: torch.full(like[k].shape, float("nan"), dtype=bf16 if k == "dx" else dtype, device="cuda") for k in names}
        binding.gated_ffn_grad(dy, x, wg, wu, wd, workspace=ws, **keep, **out)
        assert binding.layer_status(ws) == 0 and (behind == 0xA5).all(), names
        return out

    whole = run(list(like), torch.float32)
    names = list(like)
    for choice in range(1, 15):
        some = run([k for i, k in enumerate(names) if choice >> i & 1], torch.float32)
        for k, t in some.items():
            # the operands are the same bits: sums in another order, each off by the adding into the accumulator of 16 products at
            # a time (2^-23 of the sum of magnitudes), of which random terms leave sqrt(depth) in the value's own size; dx is
            # rounded to bf16 twice
            depth = 2 * m if k == "dx" else rows
            bound = (depth / 16 + 4) * 2.0**-22 * depth**0.5 + (2.0**-7 if k == "dx" else 0.0)
            assert float((t - whole[k]).float().norm() / whole[k].float().norm()) <= bound, (choice, k)
