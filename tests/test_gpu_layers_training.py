"""A run of the operators together, as a worker and the parameter server use them: lookup, linear layer, gated block with
8-bit checkpoints, logits; backward through all of them; the ragged workers' gradients through the AdamW plan, whose bf16
copy the next iteration reads."""
import pytest
import torch

import layers_reference as ref
from paper_2305_12213_b200 import binding

pytestmark = pytest.mark.gpu
bf16 = torch.bfloat16
VOCAB, WIDTH, HIDDEN, CLASSES = 500, 64, 168, 96
SHAPES = {"table": (VOCAB, WIDTH), "w_in": (WIDTH, WIDTH), "b_in": (WIDTH,), "w_gate": (WIDTH, HIDDEN), "w_up": (WIDTH, HIDDEN),
          "w_down": (HIDDEN, WIDTH), "w_out": (WIDTH, CLASSES)}


def worker_pass(p, tokens, labels):
    """One worker's gradients (bf16), its logits, and the tensors kept on the way."""
    rows = tokens.numel()
    new = lambda *s: torch.empty(*s, dtype=bf16, device="cuda")  # noqa: E731
    sizes = [binding.linear_workspace_bytes(rows, WIDTH, CLASSES), binding.linear_grad_workspace_bytes(rows, WIDTH, CLASSES),
             binding.linear_grad_workspace_bytes(rows, WIDTH, WIDTH), binding.linear_workspace_bytes(rows, WIDTH, WIDTH),
             binding.gated_ffn_workspace_bytes(rows, WIDTH, HIDDEN), binding.gated_ffn_grad_workspace_bytes(rows, WIDTH, HIDDEN),
             binding.embedding_grad_workspace_bytes(rows, VOCAB, WIDTH)]
    ws = torch.empty(max(sizes), dtype=torch.uint8, device="cuda")
    e, x, y, logits = new(rows, WIDTH), new(rows, WIDTH), new(rows, WIDTH), new(rows, CLASSES)
    binding.embedding(tokens, p["table"], e, scale=8.0)
    z = new(rows, WIDTH)
    binding.linear(e, p["w_in"], x, ws, bias=p["b_in"], activation="gelu", residual=e, z=z)
    codes = lambda: torch.empty(rows, HIDDEN, dtype=torch.float8_e4m3fn, device="cuda")  # noqa: E731
    scales = lambda: torch.empty(rows, binding.checkpoint_scales(HIDDEN), dtype=torch.float8_e8m0fnu, device="cuda")  # noqa: E731
    kept = dict(gate=codes(), up=codes(), gate_scale=scales(), up_scale=scales())
    binding.gated_ffn(x, p["w_gate"], p["w_up"], p["w_down"], y, ws, residual=x, **kept)
    binding.linear(y, p["w_out"], logits, ws)
    # the loss's own gradient: mean cross-entropy over the worker's rows
    dl = ((torch.softmax(logits.float(), 1) - torch.nn.functional.one_hot(labels.long(), CLASSES)) / rows).to(bf16)
    g = {k: new(*s) for k, s in SHAPES.items()}
    dy, dx, de = new(rows, WIDTH), new(rows, WIDTH), new(rows, WIDTH)
    binding.linear_grad(dl, y, p["w_out"], ws, dx=dy, dw=g["w_out"])
    binding.gated_ffn_grad(dy, x, p["w_gate"], p["w_up"], p["w_down"], workspace=ws, **kept, dx=dx, dw_gate=g["w_gate"],
                           dw_up=g["w_up"], dw_down=g["w_down"], dx_addend=dy)
    binding.linear_grad(dx, e, p["w_in"], ws, z=z, activation="gelu", dx=de, dw=g["w_in"], dbias=g["b_in"], dx_addend=dx)
    binding.embedding_grad(tokens, de, g["table"], ws, scale=8.0)
    return g, logits, kept, dl


def reference(p, tokens, labels, kept, dl):
    """64-bit gradients, with gate and up as they were kept and the loss's gradient as it was rounded."""
    v = {k: t.double().cpu().requires_grad_() for k, t in p.items()}
    t = tokens.cpu().long()
    e = torch.where((t >= 0)[:, None], v["table"][t.clamp_min(0)] * 8, torch.zeros((), dtype=torch.float64))
    zin = e @ v["w_in"] + v["b_in"]
    x = zin * torch.special.ndtr(zin) + e
    gate, up = x @ v["w_gate"], x @ v["w_up"]
    held = lambda z, name: z + (ref.unpack(kept[name].cpu(), kept[name + "_scale"].view(torch.uint8).cpu()) - z).detach()  # noqa: E731
    y = (torch.nn.functional.silu(held(gate, "gate")) * held(up, "up")) @ v["w_down"] + x
    logits = y @ v["w_out"]
    logits.backward(dl.double().cpu())
    return {k: t.grad for k, t in v.items()}


def test_ragged_workers_train_together():
    g = torch.Generator(device="cuda").manual_seed(1)
    params = {k: torch.empty(*s, device="cuda").normal_(0, 0.05 if k == "table" else s[0]**-0.5, generator=g) for k, s in SHAPES.items()}
    copies = {k: t.to(bf16) for k, t in params.items()}
    names, batches = list(SHAPES), [37, 200, 91]
    grads = [{k: torch.zeros(*SHAPES[k], dtype=bf16, device="cuda") for k in names} for _ in batches]
    zeros = lambda: [torch.zeros_like(params[k]) for k in names]  # noqa: E731
    plan = binding.AdamWPlan([[w[k] for k in names] for w in grads], [params[k] for k in names], zeros(), zeros(),
                             params_bf16=[copies[k] for k in names], clip=True)
    for step in (1, 2):
        for b, into in zip(batches, grads):
            tokens = torch.randint(-1, VOCAB, (b,), generator=g, device="cuda", dtype=torch.int32)
            labels = torch.randint(0, CLASSES, (b,), generator=g, device="cuda", dtype=torch.int32)
            got, logits, kept, dl = worker_pass(copies, tokens, labels)
            want = reference(copies, tokens, labels, kept, dl)
            for k in names:
                into[k].copy_(got[k])
                off = float((got[k].double().cpu() - want[k]).norm() / want[k].norm())
                # a gradient passes at most nine roundings to bf16 on its way (logits' gradient given: dy, h, d_gate, dx, z,
                # dz, de, the activation it meets, itself) of at most 2^-8 each; the 8-bit values, which the first block's
                # input meets as kept, are those of the reference
                assert off <= 9 * ref.BF16, (k, off)
        before = {k: t.clone() for k, t in params.items()}
        plan.step(batches, 1e-3, 0.9, 0.95, 1e-8, step, max_norm=1.0)
        assert all(torch.equal(copies[k], params[k].to(bf16)) and not torch.equal(params[k], before[k]) for k in names)
