"""Host threads on one AdamW or gradient-norm plan: every call has its own workers' batch sizes (CPU, the library faked)."""
import ctypes
import threading
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2305_12213_b200 import binding


@pytest.fixture
def plans(monkeypatch):
    """make(K, on_call) -> (AdamWPlan, GradNormPlan) over CPU tensors; on_call(b) stands for the library reading b."""
    fake = SimpleNamespace(db_adamw_plan_device_bytes=lambda *a: 256, db_grad_norm_plan_device_bytes=lambda *a: 256,
                           db_adamw_plan_create="create", db_grad_norm_plan_create="create",
                           db_aggregate_adamw_multi="step", db_grad_norm_multi="step")
    monkeypatch.setattr(binding, "lib", lambda: fake)
    monkeypatch.setattr(binding, "_dev_ptr", lambda t, dtype, name: None if t is None else t.data_ptr())
    monkeypatch.setattr(binding._ListPlan, "_make_table", lambda self, n, s: setattr(self, "table", torch.empty(n, dtype=torch.uint8)))
    hooks = {}

    def call(self, fn, *args, stream=None):
        if fn == "step":
            # what ctypes passes for a c_void_p argument, read as the library reads it
            hooks["on_call"](lambda: (ctypes.c_int32 * self.K).from_address(ctypes.cast(args[1], ctypes.c_void_p).value)[:])

    monkeypatch.setattr(binding._ListPlan, "_call", call)

    def make(K, on_call):
        hooks["on_call"] = on_call
        z = lambda: [torch.zeros(4)]  # noqa: E731
        grads = [z() for _ in range(K)]
        return binding.AdamWPlan(grads, z(), z(), z()), binding.GradNormPlan(grads)

    return make


def _step(plan, b):
    if isinstance(plan, binding.AdamWPlan):
        plan.step(b, 1e-3, 0.9, 0.999, 1e-8, 1)
    else:
        plan.run(b, torch.zeros(1))


@pytest.mark.parametrize("which", [0, 1])
def test_a_call_keeps_its_batch_sizes_while_another_thread_calls(plans, which):
    """Thread A has handed over its batch sizes and the library has not read them when thread B calls: A's are still A's."""
    seen, a_in, b_done = {}, threading.Event(), threading.Event()

    def on_call(read):
        if threading.current_thread().name == "A":
            a_in.set()
            assert b_done.wait(10)
        seen[threading.current_thread().name] = read()

    plan = plans(3, on_call)[which]
    a = threading.Thread(target=_step, args=(plan, [1, 2, 3]), name="A")
    a.start()
    assert a_in.wait(10)
    b = threading.Thread(target=_step, args=(plan, [70, 0, 5]), name="B")
    b.start()
    b.join(10)
    b_done.set()
    a.join(10)
    assert seen == {"A": [1, 2, 3], "B": [70, 0, 5]}

@pytest.mark.parametrize("which", [0, 1])
def test_batch_sizes_of_any_integer_type_and_none_that_does_not_fit(plans, which):
    got = []
    plan = plans(2, lambda read: got.append(read()))[which]
    for b in ([3, 4], (3, 4), np.array([3, 4]), [np.int64(3), np.int32(4)]):
        _step(plan, b)
    assert got == [[3, 4]] * 4
    for bad in ([2**31, 1], [2**32 + 3, 4], [-(2**31) - 1, 1]):         # none is cut to 32 bits and taken
        with pytest.raises(ValueError):
            _step(plan, bad)
    with pytest.raises(TypeError):
        _step(plan, [1.5, 2])
    with pytest.raises(ValueError):
        _step(plan, [1])
    assert len(got) == 4
