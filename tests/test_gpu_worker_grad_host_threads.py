"""The worker gradient and the general contraction from a host thread whose first CUDA call they are: the same bits as from the
main thread."""
import threading

import pytest
import torch

from paper_2305_12213_b200 import binding, inputs

pytestmark = pytest.mark.gpu
DEV = "cuda"


def in_new_thread(body):
    failed = []

    def run():
        try:
            body()
        except BaseException as e:  # noqa: BLE001
            failed.append(e)

    t = threading.Thread(target=run)
    t.start()
    t.join()
    torch.cuda.synchronize()
    if failed:
        raise failed[0]


@pytest.mark.parametrize("b_i,D,C", [(24, 256, 100), (128, 2048, 1000)])
def test_worker_gradient(b_i, D, C):
    X, y, W = inputs.softmax_problem([b_i], D, C, seed=7, w_std=0.05, device=DEV)
    stream = torch.cuda.current_stream()
    ws = torch.empty(binding.worker_grad_workspace_bytes(b_i, D, C), dtype=torch.uint8, device=DEV)
    here, there = torch.zeros(D, C, device=DEV), torch.zeros(D, C, device=DEV)
    in_new_thread(lambda: binding.worker_grad(X, y, W, there, None, ws, stream=stream))
    binding.worker_grad(X, y, W, here, None, ws)
    assert torch.equal(here, there) and float(here.abs().max()) > 0


def test_grouped_worker_gradients():
    offsets, D, C = [0, 24, 64, 128, 256], 256, 100
    X, y, W = inputs.softmax_problem([24, 40, 64, 128], D, C, seed=8, w_std=0.05, device=DEV)
    stream = torch.cuda.current_stream()
    ws = torch.empty(binding.worker_grad_grouped_workspace_bytes(256, 4, D, C), dtype=torch.uint8, device=DEV)
    here, there = ([torch.zeros(D, C, device=DEV) for _ in range(4)] for _ in range(2))
    in_new_thread(lambda: binding.worker_grad_grouped(X, y, W, offsets, there, None, ws, stream=stream))
    binding.worker_grad_grouped(X, y, W, offsets, here, None, ws)
    assert all(torch.equal(a, b) and float(a.abs().max()) > 0 for a, b in zip(here, there))


def test_contraction():
    A, B = torch.randn(96, 512, device=DEV), torch.randn(200, 512, device=DEV)
    stream = torch.cuda.current_stream()
    here, there = torch.zeros(96, 200, device=DEV), torch.zeros(96, 200, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    in_new_thread(lambda: binding.contract_f32(A, B, there, status, stream=stream))
    in_new_thread(lambda: binding.contract_f32(A, B.t().contiguous().t(), there, status, stream=stream))
    binding.contract_f32(A, B.t().contiguous().t(), here, status)
    assert torch.equal(here, there) and float(here.abs().max()) > 0 and int(status.item()) == 0
