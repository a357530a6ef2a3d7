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
