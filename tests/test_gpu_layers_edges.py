"""Calls of the layers that their documentation allows and that are easily got wrong: buffers at any element of a flat one, offsets
past 32 bits, scales that are not finite, in-place sums and rows that are not finite in the kernels of CTA pairs."""
import pytest
import torch

import layers_reference as ref
from paper_2305_12213_b200 import binding
from test_gpu_layers import bf16, e4m3, e8m0, f64, gen, kept_buffers, normal, workspace

pytestmark = pytest.mark.gpu


def at(t, shift):
    """The same values, contiguous, `shift` elements behind a 256-byte boundary."""
    raw = t.view(torch.uint8) if t.element_size() == 1 else t
    flat = torch.zeros(raw.numel() + 256, dtype=raw.dtype, device="cuda")
    out = flat[shift:shift + raw.numel()].view(raw.shape)
    out.copy_(raw)
    return out.view(t.dtype)


@pytest.mark.parametrize("shift", [1, 3, 8])
@pytest.mark.parametrize("kept", ["bf16", "e4m3"])
@pytest.mark.parametrize("rows,n,m", [(130, 72, 200), (67, 33, 70)])
def test_every_buffer_at_any_element(rows, n, m, kept, shift):
    """Operands and results as parts of flat buffers, off every grid: the same bits as on it."""
    x, w, b, r, dy = normal(1, rows, n), normal(2, n, m, std=0.1), normal(3, m), normal(4, rows, m), normal(5, rows, m)
    add, wd, ry = normal(6, rows, n), normal(7, m, n, std=0.1), normal(8, rows, n)
    size = max(f(rows, n, m, aligned=False) for f in (binding.linear_workspace_bytes, binding.linear_grad_workspace_bytes,
                                                      binding.gated_ffn_workspace_bytes, binding.gated_ffn_grad_workspace_bytes))
    ws = workspace(size)

    def run(put):
        keep = {k: put(t) for k, t in kept_buffers(rows, m, kept, ["z"]).items()}
        both = {k: put(t) for k, t in kept_buffers(rows, m, kept, ["gate", "up"]).items()}
        new = lambda dtype, *s: put(torch.zeros(*s, dtype=dtype, device="cuda"))  # noqa: E731
        out = {"y": new(bf16, rows, m), "dx": new(bf16, rows, n), "dw": new(torch.float32, n, m), "db": new(torch.float32, m),
               "dw16": new(bf16, n, m), "db16": new(bf16, m), "fy": new(bf16, rows, n), "fdx": new(bf16, rows, n),
               "fg": new(bf16, n, m), "fu": new(bf16, n, m), "fd": new(bf16, m, n)}
        xs, ws_, bs, rs, dys = put(x), put(w), put(b), put(r), put(dy)
        binding.linear(xs, ws_, out["y"], ws, bias=bs, residual=rs, activation="silu", **keep)
        binding.linear_grad(dys, xs, ws_, ws, activation="silu", **keep, dx=out["dx"], dw=out["dw"], dbias=out["db"], dx_addend=put(add))
        binding.linear_grad(dys, xs, ws_, ws, activation="silu", **keep, dw=out["dw16"], dbias=out["db16"])
        binding.gated_ffn(xs, ws_, ws_, put(wd), out["fy"], ws, residual=put(ry), activation="gelu", **both)
        binding.gated_ffn_grad(put(ry), xs, ws_, ws_, put(wd), workspace=ws, activation="gelu", **both, dx=out["fdx"],
                               dw_gate=out["fg"], dw_up=out["fu"], dw_down=out["fd"])
        assert binding.layer_status(ws) == 0
        return {**out, **keep, **both}

    want, got = run(lambda t: t.clone()), run(lambda t: at(t, shift))
    bits = lambda t: t.contiguous().view(torch.uint8)  # noqa: E731
    for k in want:
        assert torch.equal(bits(got[k]), bits(want[k])), k


@pytest.mark.parametrize("act,kept", [("relu", "e4m3"), ("gelu", "bf16"), ("silu", "e4m3")])
def test_bias_gradient_alone_behind_an_activation(act, kept):
    rows, n, m = 333, 40, 300
    x, w, dy = normal(1, rows, n), normal(2, n, m, std=0.2), normal(3, rows, m)
    keep = kept_buffers(rows, m, kept, ["z"])
    ws = workspace(max(binding.linear_workspace_bytes(rows, n, m), binding.linear_grad_workspace_bytes(rows, n, m)))
    binding.linear(x, w, torch.empty(rows, m, dtype=bf16, device="cuda"), ws, activation=act, **keep)
    with_dw, alone = torch.empty(m, device="cuda"), torch.zeros(m, device="cuda")
    binding.linear_grad(dy, x, w, ws, activation=act, **keep, dbias=with_dw, dw=torch.empty(n, m, device="cuda"))
    binding.linear_grad(dy, None, w, ws, activation=act, **keep, dbias=alone)
    assert torch.equal(alone, with_dw)


PAIRS = (2050, 1096, 2184)              # pairs of CTAs in every product (test_layers_plan)


def test_in_place_and_columns_in_the_kernels_of_pairs():
    rows, n, m = PAIRS
    wide = normal(1, rows, n + m + n + 40)
    x, r = wide[:, :n], normal(2, rows, m)
    w, dy, add = normal(3, n, m, std=0.03), normal(4, rows, m), normal(5, rows, n)
    ws = workspace(max(binding.linear_workspace_bytes(rows, n, m), binding.linear_grad_workspace_bytes(rows, n, m)))
    y, dx = torch.empty_like(r), torch.empty_like(add)
    binding.linear(x.contiguous(), w, y, ws, residual=r, activation="gelu")
    binding.linear_grad(dy, None, w, ws, dx=dx, dx_addend=add)
    before = wide.clone()
    wide[:, n:n + m].copy_(r)
    wide[:, n + m + 8:n + m + 8 + n].copy_(add)
    binding.linear(x, w, wide[:, n:n + m], ws, residual=wide[:, n:n + m], activation="gelu")
    binding.linear_grad(dy, None, w, ws, dx=wide[:, n + m + 8:n + m + 8 + n], dx_addend=wide[:, n + m + 8:n + m + 8 + n])
    before[:, n:n + m], before[:, n + m + 8:n + m + 8 + n] = y, dx
    assert torch.equal(wide, before)


def test_rows_that_are_not_finite_in_the_kernels_of_pairs():
    rows, n, m = PAIRS
    x, wg, wu, wd = normal(1, rows, n), normal(2, n, m, std=0.03), normal(3, n, m, std=0.03), normal(4, m, n, std=0.02)
    dy = normal(5, rows, n)
    ws = workspace(max(binding.gated_ffn_workspace_bytes(rows, n, m), binding.gated_ffn_grad_workspace_bytes(rows, n, m)))

    def run():
        keep = kept_buffers(rows, m, "e4m3", ["gate", "up"])
        y, dx = torch.empty_like(x), torch.empty_like(x)
        binding.gated_ffn(x, wg, wu, wd, y, ws, **keep)
        binding.gated_ffn_grad(dy, x, wg, wu, wd, workspace=ws, **keep, dx=dx)
        return y, dx, keep["gate"].float(), keep["up"].float()

    clean = run()
    touched = [0, 127, 128, 255, 1000, rows - 1]
    for i, v in zip(touched, [float("nan"), float("inf"), float("-inf")] * 2):
        x[i, (37 * i) % n] = v
    others = torch.ones(rows, dtype=torch.bool, device="cuda")
    others[touched] = False
    for was, now in zip(clean, run()):
        assert torch.equal(was[others], now[others])
        assert not now[touched].isfinite().all(1).any()


@pytest.mark.parametrize("rows,n,m", [PAIRS, (256, 2048, 1000), (333, 1001, 777)])
def test_same_bits_again_replayed_and_beside_another_stream(rows, n, m):
    x, w, b, dy = normal(1, rows, n), normal(2, n, m, std=n**-0.5), normal(3, m), normal(4, rows, m)
    wd, dyn = normal(5, m, n, std=m**-0.5), normal(6, rows, n)
    size = max(f(rows, n, m) for f in (binding.linear_workspace_bytes, binding.linear_grad_workspace_bytes,
                                       binding.gated_ffn_workspace_bytes, binding.gated_ffn_grad_workspace_bytes))

    def buffers():
        new = lambda *s: torch.zeros(*s, dtype=bf16, device="cuda")  # noqa: E731
        return (workspace(size), {**kept_buffers(rows, m, "e4m3", ["z"])}, kept_buffers(rows, m, "bf16", ["gate", "up"]),
                dict(y=new(rows, m), dx=new(rows, n), dw=new(n, m), db=new(m), fy=new(rows, n), fdx=new(rows, n), fg=new(n, m),
                     fu=new(n, m), fd=new(m, n)))

    def step(ws, z, both, o):
        binding.linear(x, w, o["y"], ws, bias=b, activation="silu", **z)
        binding.linear_grad(dy, x, w, ws, activation="silu", **z, dx=o["dx"], dw=o["dw"], dbias=o["db"])
        binding.gated_ffn(x, w, w, wd, o["fy"], ws, residual=x, **both)
        binding.gated_ffn_grad(dyn, x, w, w, wd, workspace=ws, **both, dx=o["fdx"], dw_gate=o["fg"], dw_up=o["fu"], dw_down=o["fd"],
                               dx_addend=dyn)

    first, second, third = buffers(), buffers(), buffers()
    step(*first)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*third)
    for t in third[3].values():
        t.fill_(3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(side):
            step(*second)
        graph.replay()
    torch.cuda.synchronize()
    for other in (second, third):
        assert binding.layer_status(other[0]) == 0
        for k, t in first[3].items():
            assert torch.equal(t.view(torch.int16), other[3][k].view(torch.int16)), k


# ------------------------------------------------------------------------------------------------ offsets past 32 bits
FAR = (60000, 40000)                    # a tensor of 2.4 * 10^9 elements whose columns are the operands


def far(dtype, cols, shift, seed):
    wide = torch.empty(*FAR, dtype=dtype, device="cuda")
    t = wide[:, shift:shift + cols]
    t.copy_(normal(seed, FAR[0], cols).to(dtype))
    return t


def test_layers_far_from_their_first_row():
    rows, n, m = FAR[0], 64, 136
    w, wg, wd = normal(1, n, m, std=0.1), normal(2, n, m, std=0.1), normal(3, m, n, std=0.1)
    size = max(f(rows, n, m, aligned=False) for f in (binding.linear_workspace_bytes, binding.linear_grad_workspace_bytes,
                                                      binding.gated_ffn_workspace_bytes, binding.gated_ffn_grad_workspace_bytes))
    ws = workspace(size)
    for shift in (8, 3):                                        # on the grid, and copied onto it
        x, y = far(bf16, n, shift, 4), far(bf16, m, 1000 + shift, 5)
        near_x, near_y = x.contiguous(), torch.empty(rows, m, dtype=bf16, device="cuda")
        binding.linear(x, w, y, ws, residual=y, activation="silu")
        binding.linear(near_x, w, near_y, ws, residual=normal(5, rows, m), activation="silu")
        assert torch.equal(y, near_y)
        dx, near_dx, dw, near_dw = far(bf16, n, 2000, 6), torch.empty_like(near_x), torch.empty_like(w), torch.empty_like(w)
        binding.linear_grad(y, x, w, ws, dx=dx, dw=dw)
        binding.linear_grad(near_y, near_x, w, ws, dx=near_dx, dw=near_dw)
        assert torch.equal(dx, near_dx) and torch.equal(dw, near_dw)
        binding.gated_ffn(x, w, wg, wd, dx, ws, residual=x)
        binding.gated_ffn(near_x, w, wg, wd, near_dx, ws, residual=near_x)
        assert torch.equal(dx, near_dx)
        del x, y, dx


def test_checkpoints_and_embedding_far_from_their_first_row():
    rows, n = FAR[0], 72
    x = far(bf16, n, 8, 1)
    codes = torch.zeros(rows, n, dtype=torch.uint8, device="cuda").view(e4m3)
    scale = torch.zeros(rows, binding.checkpoint_scales(n), dtype=torch.uint8, device="cuda").view(e8m0)
    binding.checkpoint_pack(x, codes, scale)
    want_codes, want_scale = ref.pack(x[-100:].float().cpu())
    assert torch.equal(scale[-100:].view(torch.uint8).cpu(), want_scale)
    assert torch.equal(codes[-100:].view(torch.uint8).cpu(), want_codes.view(torch.uint8))
    binding.checkpoint_unpack(codes, scale, x)
    assert torch.equal(x[-100:].cpu(), ref.unpack(want_codes, want_scale).float().to(bf16))
    tokens = torch.randint(-1, 301, (rows,), generator=gen(2), device="cuda", dtype=torch.int32)
    table = normal(3, 300, n)
    binding.embedding(tokens, table, x)
    near = torch.empty(rows, n, dtype=bf16, device="cuda")
    binding.embedding(tokens, table, near)
    assert torch.equal(x, near)
    ws = workspace(binding.embedding_grad_workspace_bytes(rows, 300, n))
    got, want = torch.empty(300, n, device="cuda"), torch.empty(300, n, device="cuda")
    binding.embedding_grad(tokens, x, got, ws)
    binding.embedding_grad(tokens, near, want, ws)
    assert torch.equal(got, want)


def test_whole_tensors_past_32_bits():
    """More than 2^32 bytes of codes and of a table's rows, in one piece."""
    rows, n = 34000, 131072
    x = torch.empty(rows, n, dtype=bf16, device="cuda")
    x.copy_(normal(1, 1, n).expand(rows, n))
    x[-1] = normal(2, 1, n)[0]
    codes = torch.zeros(rows, n, dtype=torch.uint8, device="cuda").view(e4m3)
    scale = torch.zeros(rows, n // 32, dtype=torch.uint8, device="cuda").view(e8m0)
    binding.checkpoint_pack(x, codes, scale)
    for i in (0, rows // 2, rows - 1):
        want_codes, want_scale = ref.pack(x[i:i + 1].float().cpu())
        assert torch.equal(codes[i:i + 1].view(torch.uint8).cpu(), want_codes.view(torch.uint8))
        assert torch.equal(scale[i:i + 1].view(torch.uint8).cpu(), want_scale)
    x.zero_()
    binding.checkpoint_unpack(codes, scale, x)
    assert torch.equal(x[-1:].cpu(), ref.unpack(codes[-1:].cpu(), scale[-1:].view(torch.uint8).cpu()).float().to(bf16))
    # the last row of a table of that size, looked up and summed into
    tokens = torch.tensor([rows - 1, 0, -1, rows - 1] * 70, dtype=torch.int32, device="cuda")
    out = torch.empty(280, n, dtype=bf16, device="cuda")
    binding.embedding(tokens, x, out)
    assert torch.equal(out[-1], x[-1]) and torch.equal(out[1], x[0]) and (out[2] == 0).all()
    last = x[-1].float()
    x.fill_(5)
    ws = workspace(binding.embedding_grad_workspace_bytes(280, rows, n))
    binding.embedding_grad(tokens, out, x, ws, scale=1 / 128)
    want = 140 / 128 * last                                     # 140 equal terms: each sum is off by half a step of fp32
    assert ((x[-1].float() - want).abs() <= (ref.BF16 + 141 * 2.0**-24) * want.abs()).all()
    assert (x[1:-1] == 0).all()


# ------------------------------------------------------------------------------------------------ scales
@pytest.mark.parametrize("scale", [float("inf"), float("nan"), -2.0, 0.0])
@pytest.mark.parametrize("rows", [40, 700])
def test_rows_without_a_token_are_zeros_whatever_the_scale(rows, scale):
    vocab, n = 90, 24
    tokens = torch.randint(0, vocab // 2, (rows,), generator=gen(1), device="cuda", dtype=torch.int32) * 2 - 1     # -1, 1, 3, ...
    table, dy = normal(2, vocab, n, dtype=torch.float32), normal(3, rows, n, dtype=torch.float32)
    out = torch.full((rows, n), 7.0, device="cuda")
    binding.embedding(tokens, table, out, scale=scale)
    t = tokens.cpu().long()
    want = torch.where((t >= 0)[:, None], table.cpu()[t.clamp_min(0)] * scale, torch.zeros(()))
    assert torch.equal(out.cpu().nan_to_num(1e9), want.nan_to_num(1e9))
    assert (out.view(torch.int32)[tokens < 0] == 0).all()
    grad = torch.full((vocab, n), 7.0, device="cuda")
    binding.embedding_grad(tokens, dy, grad, workspace(binding.embedding_grad_workspace_bytes(rows, vocab, n)), scale=scale)
    used = torch.zeros(vocab, dtype=torch.bool, device="cuda")
    used[tokens[tokens >= 0].long()] = True
    assert (grad.view(torch.int32)[~used] == 0).all()
    if scale != scale or scale in (float("inf"),):
        assert not grad[used].isfinite().any()
    else:
        want = ref.embedding_grad(tokens, dy.cpu(), vocab, scale)
        size = ref.embedding_grad(tokens, dy.cpu().abs(), vocab, abs(scale))
        assert ((f64(grad) - want).abs() <= (rows + 2) * 2.0**-24 * size + 1e-300).all()
