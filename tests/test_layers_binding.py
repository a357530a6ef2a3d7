"""What the layers' binding refuses before anything is enqueued, on the CPU: its helpers take the device of a tensor as an index, and
a CPU tensor's is -1."""
import pytest
import torch

from paper_2305_12213_b200 import binding

CPU = -1


def test_workspace_that_is_not_its_memory():
    whole = torch.zeros(4096, dtype=torch.uint8)
    assert binding._scratch(whole, CPU) == (whole.data_ptr(), 4096)
    for view in (torch.zeros(1, dtype=torch.uint8).expand(4096), whole[::2], whole.view(64, 64).t()):
        with pytest.raises(TypeError):                          # one byte expanded to 4096 would be written far past its end
            binding._scratch(view, CPU)
    with pytest.raises(ValueError):
        binding._scratch(whole, 0)
