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


class _Recorded:
    """Stands for the library: keeps the arguments as the C side would see them."""

    def __init__(self, monkeypatch):
        self.seen = {}
        monkeypatch.setattr(binding, "lib", lambda: self)
        monkeypatch.setattr(binding, "_device_index", lambda t: CPU)
        monkeypatch.setattr(binding, "_launch", lambda index, stream, fn, *args: fn(*args, 0))

    def __getattr__(self, name):
        def call(*args):
            self.seen[name] = [t(a).value if t is not binding.c_void_p else a for t, a in zip(binding._SIGNATURES[name][1], args)]
            return 0
        return call


def huge(rows, cols, dtype=torch.bfloat16):
    """[rows, cols] without memory behind it: shape, type and strides are all that a check looks at."""
    return torch.empty(rows, cols, dtype=dtype, device="meta")


@pytest.mark.parametrize("n", [2**31, 2**32 + 8, 2**33 + 1])
def test_sizes_past_32_bits_do_not_become_others(monkeypatch, n):
    """2^32 + 8 features would reach the C side as 8."""
    lib = _Recorded(monkeypatch)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: CPU)
    monkeypatch.setattr(torch.Tensor, "data_ptr", lambda t: 4096)
    ws, bf = torch.empty(16, dtype=torch.uint8), torch.bfloat16
    codes, scale = huge(1, n, torch.float8_e4m3fn), huge(1, binding.checkpoint_scales(n), torch.float8_e8m0fnu)
    tokens = torch.empty(1, dtype=torch.int32)
    binding.linear(huge(1, n), huge(n, 8), huge(1, 8), ws)
    assert lib.seen["db_linear"].count(-1) == 1
    binding.linear(huge(1, 8), huge(8, n), huge(1, n), ws)
    assert lib.seen["db_linear"].count(-1) == 1
    binding.linear_grad(huge(1, n), None, huge(8, n), ws, dx=huge(1, 8))
    assert lib.seen["db_linear_grad"].count(-1) == 1
    binding.linear_grad(huge(1, 8), huge(1, n), huge(n, 8), ws, dw=huge(n, 8))
    assert lib.seen["db_linear_grad"].count(-1) == 1
    for width, hidden in ((n, 8), (8, n)):
        up, down, x, h = huge(width, hidden), huge(hidden, width), huge(1, width), huge(1, hidden)
        binding.gated_ffn(x, up, up, down, x, ws)
        assert lib.seen["db_gated_ffn"].count(-1) == 1
        binding.gated_ffn_grad(x, x, up, up, down, h, h, ws, dx=x)
        assert lib.seen["db_gated_ffn_grad"].count(-1) == 1
    binding.checkpoint_pack(huge(1, n), codes, scale)
    binding.checkpoint_unpack(codes, scale, huge(1, n))
    assert lib.seen["db_checkpoint_pack"].count(-1) == lib.seen["db_checkpoint_unpack"].count(-1) == 1
    for vocab, width in ((n, 8), (8, n)):
        binding.embedding(tokens, huge(vocab, width), huge(1, width))
        binding.embedding_grad(tokens, huge(1, width), huge(vocab, width), ws)
        assert lib.seen["db_embedding"].count(-1) == lib.seen["db_embedding_grad"].count(-1) == 1


def test_workspace_queries_of_sizes_past_their_type():
    for f in (binding.linear_workspace_bytes, binding.linear_grad_workspace_bytes, binding.gated_ffn_workspace_bytes,
              binding.gated_ffn_grad_workspace_bytes, binding.embedding_grad_workspace_bytes):
        assert f(8, 8, 8) > 0
        for bad in ((2**64 + 8, 8, 8), (-2**64 + 8, 8, 8), (8, 2**32 + 8, 8), (8, 8, 2**32 + 8), (8, -2**32 + 8, 8)):
            assert f(*bad) == 0, bad
    # any truth value says that operands are aligned
    assert binding.linear_workspace_bytes(100, 64, 64, 2**32) == binding.linear_workspace_bytes(100, 64, 64, True)
