"""Linear layer, gated feed-forward block, 8-bit checkpoints and embedding table on the GPU against 64 bits.

Bounds: products of bf16 are exact in fp32; 16 of them at a time are added into an accumulator that truncates
(layers_reference.product_bound); an output, and an operand that is itself a result, is rounded to bf16 once (2^-8
relative); the fast exponential and quotient are within 2^-20.  Each bound holds for every element, for any order of sums."""
import pytest
import torch

import layers_reference as ref
from paper_2305_12213_b200 import binding

pytestmark = pytest.mark.gpu
BF16, FAST = ref.BF16, 2.0**-20
bf16, e4m3, e8m0 = torch.bfloat16, torch.float8_e4m3fn, torch.float8_e8m0fnu


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(seed, *shape, std=1.0, dtype=bf16, pitch=0, shift=0):
    """[rows, cols] normal values; pitch > 0: rows of a wider tensor, `shift` elements off its start."""
    g = gen(seed)
    if not pitch:
        return (torch.empty(*shape, device="cuda").normal_(0, std, generator=g)).to(dtype)
    wide = torch.empty(shape[0], pitch, device="cuda").normal_(0, std, generator=g).to(dtype)
    return wide[:, shift:shift + shape[1]]


def f64(t):
    return t.detach().float().cpu().double()


def within(got, want, bound):
    got = f64(got)
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), (f"{int(bad.sum())} of {bad.numel()} outside, worst by a factor "
                           f"{float(((got - want).abs() / bound.clamp_min(1e-300))[bad].max()):.3g}")
    # independent roundings add up like their squares: two of at most 2^-8 stay below 2^-7 of the norm
    if float(want.norm()) > 0:
        assert float((got - want).norm() / want.norm()) <= 2.0**-7


def kept_buffers(rows, n, kept, names):
    if kept == "none":
        return {}
    if kept == "bf16":
        return {k: torch.full((rows, n), float("nan"), dtype=bf16, device="cuda") for k in names}
    out = {k: torch.zeros(rows, n, dtype=torch.uint8, device="cuda").view(e4m3) for k in names}
    out.update({k + "_scale": torch.zeros(rows, -(-n // 32), dtype=torch.uint8, device="cuda").view(e8m0) for k in names})
    return out


def kept_values(kept, name):
    t = kept[name]
    if t.dtype == bf16:
        return f64(t)
    return ref.unpack(t.cpu(), kept[name + "_scale"].view(torch.uint8).cpu())


def check_kept(kept, name, z, bound):
    """What was kept of z lies within half a step of a value within `bound` of z."""
    got = kept_values(kept, name)
    if kept[name].dtype == bf16:
        assert ((got - z).abs() <= BF16 * z.abs() + (1 + BF16) * bound).all()
        return
    scale = torch.exp2(kept[name + "_scale"].view(torch.uint8).cpu().double() - 127)
    step = scale.repeat_interleave(32, 1)[:, :z.shape[1]]
    assert ((got - z).abs() <= torch.maximum(2.0**-4 * z.abs(), 2.0**-10 * step) + (1 + 2.0**-4) * bound).all()
    # each scale is the smallest that holds its group, up to the error of the group's largest value
    groups = scale.shape[1] * 32
    pad = lambda t: torch.nn.functional.pad(t, (0, groups - t.shape[1])).view(t.shape[0], -1, 32)  # noqa: E731
    top, slack = pad(z.abs()).amax(2), pad(bound).amax(2)
    assert (top - slack <= 448 * scale).all()
    assert ((top + slack > 224 * scale) | (scale <= 2.0**-127)).all()


def workspace(nbytes):
    return torch.full((nbytes + 256,), 0xA5, dtype=torch.uint8, device="cuda")[:nbytes]


LINEAR = [  # rows, n_in, n_out, bias, residual, activation, kept, pitch, shift
    (1, 64, 64, True, True, "none", "bf16", 0, 0),
    (1, 1, 1, True, False, "relu", "bf16", 0, 0),
    (7, 8, 24, False, True, "gelu", "e4m3", 0, 0),
    (129, 64, 72, True, False, "silu", "e4m3", 96, 16),
    (128, 256, 128, False, False, "none", "none", 0, 0),
    (300, 512, 264, True, True, "gelu", "bf16", 0, 0),
    (255, 100, 33, True, True, "silu", "bf16", 0, 0),
    (77, 33, 100, False, False, "relu", "e4m3", 0, 0),
    (64, 64, 64, True, True, "silu", "bf16", 80, 3),        # rows that start off the 16-byte grid
    (200, 2048, 1000, True, False, "none", "bf16", 0, 0),   # reduction split, classes no multiple of 32
    (1000, 72, 2056, True, True, "gelu", "e4m3", 72, 0),
    (1025, 1032, 520, False, True, "silu", "e4m3", 0, 0),
    (4100, 320, 640, True, True, "gelu", "bf16", 0, 0),     # pairs of CTAs, several tiles each
]


@pytest.mark.parametrize("rows,n,m,bias,residual,act,kept,pitch,shift", LINEAR)
def test_linear(rows, n, m, bias, residual, act, kept, pitch, shift):
    x = normal(1, rows, n, pitch=pitch, shift=shift)
    w, b = normal(2, n, m, std=n**-0.5), normal(3, m, std=0.5) if bias else None
    r = normal(4, rows, m) if residual else None
    keep = kept_buffers(rows, m, kept, ["z"])
    aligned = x.data_ptr() % 16 == 0 and x.stride(0) % 8 == 0 and m % 8 == 0 and n % 8 == 0
    ws = workspace(max(binding.linear_workspace_bytes(rows, n, m, aligned), binding.linear_grad_workspace_bytes(rows, n, m, aligned)))
    guard = torch.full((rows + 2, m + 8), 7.0, dtype=bf16, device="cuda")    # y is a slice: nothing around it is written
    y = guard[1:rows + 1, :m]
    binding.linear(x, w, y, ws, bias=b, residual=r, activation=act, **keep)
    assert binding.layer_status(ws) == 0
    xd, wd = f64(x), f64(w)
    z = xd @ wd + (f64(b) if bias else 0)
    off = ref.product_bound(xd, wd) + ref.ADD * z.abs()
    y64 = ref.act(z, act) + (f64(r) if residual else 0)
    # the activations' slopes stay below 1.13
    within(y, y64, BF16 * y64.abs() + (1 + BF16) * (1.13 * off + FAST * (1 + z.abs())))
    assert (guard[0] == 7).all() and (guard[-1] == 7).all() and (guard[:, m:] == 7).all()
    if kept != "none":
        check_kept(keep, "z", z, off)

    if act != "none" and kept == "none":
        return
    dy = normal(5, rows, m, pitch=pitch and m + 24, shift=shift)
    zk = kept_values(keep, "z") if kept != "none" else z
    dz = f64(dy) * ref.slope(zk, act)
    add = normal(6, rows, n) if residual else None
    for dtype in (bf16, torch.float32):
        dx = torch.full((rows, n), float("nan"), dtype=bf16, device="cuda")
        dw, db = torch.full((n, m), float("nan"), dtype=dtype, device="cuda"), torch.full((m,), float("nan"), dtype=dtype, device="cuda")
        binding.linear_grad(dy, x, w, ws, activation=act, **(keep if act != "none" else {}), dx=dx, dw=dw, dbias=db, dx_addend=add)
        assert binding.layer_status(ws) == 0
        rounded = 0.0 if act == "none" else BF16 + 2 * FAST                   # dz itself
        out = 0.0 if dtype == torch.float32 else BF16
        want = dz @ wd.T + (f64(add) if residual else 0)
        within(dx, want, BF16 * want.abs() + (1 + BF16) * ref.product_bound(dz, wd.T, rounded) + 1e-30)
        want = xd.T @ dz
        within(dw, want, out * want.abs() + (1 + out) * ref.product_bound(xd.T, dz, rounded) + 1e-30)
        # column sums: fp32, in three stages, of unrounded values
        want = dz.sum(0)
        within(db, want, out * want.abs() + (1 + out) * (rows + 4) * 2.0**-24 * dz.abs().sum(0) + 4 * FAST * f64(dy).abs().sum(0) + 1e-30)


def test_linear_gradients_one_by_one_and_in_place():
    rows, n, m = 130, 64, 96
    x, w, dy, r = normal(1, rows, n), normal(2, n, m, std=0.1), normal(3, rows, m), normal(4, rows, n)
    ws = workspace(binding.linear_grad_workspace_bytes(rows, n, m))
    whole = {"dx": torch.empty_like(x), "dw": torch.empty_like(w), "dbias": torch.empty(m, dtype=bf16, device="cuda")}
    binding.linear_grad(dy, x, w, ws, **whole)
    for name, t in whole.items():
        alone = torch.zeros_like(t)
        binding.linear_grad(dy, x if name == "dw" else None, w, ws, **{name: alone})
        assert torch.equal(alone, t), name
    apart, same = torch.empty_like(x), r.clone()
    binding.linear_grad(dy, x, w, ws, dx=apart, dx_addend=r)
    binding.linear_grad(dy, x, w, ws, dx=same, dx_addend=same)
    assert torch.equal(apart, same)
    y, same = torch.empty(rows, m, dtype=bf16, device="cuda"), dy.clone()
    wf = workspace(binding.linear_workspace_bytes(rows, n, m))
    binding.linear(x, w, y, wf, residual=dy, activation="silu")
    binding.linear(x, w, same, wf, residual=same, activation="silu")
    assert torch.equal(y, same)


FFN = [  # rows, width, hidden, residual, activation, kept, pitch, shift
    (1, 64, 128, True, "silu", "bf16", 0, 0),
    (1, 1, 1, True, "gelu", "e4m3", 0, 0),
    (100, 64, 256, True, "silu", "bf16", 0, 0),
    (130, 72, 200, False, "gelu", "e4m3", 88, 8),
    (33, 40, 33, True, "silu", "bf16", 0, 0),
    (65, 31, 70, False, "gelu", "e4m3", 0, 0),
    (64, 64, 128, True, "silu", "e4m3", 70, 1),
    (511, 136, 512, True, "relu", "bf16", 0, 0),
    (257, 128, 264, True, "none", "bf16", 0, 0),
    (1030, 512, 1032, True, "silu", "e4m3", 0, 0),
    (4097, 256, 1024, False, "gelu", "bf16", 0, 0),
]


@pytest.mark.parametrize("rows,n,m,residual,act,kept,pitch,shift", FFN)
def test_gated_ffn(rows, n, m, residual, act, kept, pitch, shift):
    x = normal(1, rows, n, pitch=pitch, shift=shift)
    wg, wu, wd = normal(2, n, m, std=n**-0.5), normal(3, n, m, std=n**-0.5), normal(4, m, n, std=m**-0.5)
    r = normal(5, rows, n) if residual else None
    keep = kept_buffers(rows, m, kept, ["gate", "up"])
    aligned = x.data_ptr() % 16 == 0 and x.stride(0) % 8 == 0 and m % 8 == 0 and n % 8 == 0
    ws = workspace(max(binding.gated_ffn_workspace_bytes(rows, n, m, aligned), binding.gated_ffn_grad_workspace_bytes(rows, n, m, aligned)))
    y = torch.full((rows, n), float("nan"), dtype=bf16, device="cuda")
    binding.gated_ffn(x, wg, wu, wd, y, ws, residual=r, activation=act, **keep)
    assert binding.layer_status(ws) == 0
    without = torch.empty_like(y)
    binding.gated_ffn(x, wg, wu, wd, without, ws, residual=r, activation=act)
    assert torch.equal(without, y)                                            # keeping changes nothing
    xd, wgd, wud, wdd = f64(x), f64(wg), f64(wu), f64(wd)
    g, u = xd @ wgd, xd @ wud
    og, ou = ref.product_bound(xd, wgd), ref.product_bound(xd, wud)
    check_kept(keep, "gate", g, og)
    check_kept(keep, "up", u, ou)
    a = ref.act(g, act)
    h = a * u
    off_a = 1.13 * og + FAST * (1 + g.abs())
    off_h = off_a * (u.abs() + ou) + a.abs() * ou
    off_h = BF16 * (h.abs() + off_h) + off_h                                   # h is rounded for the second product
    y64 = h @ wdd + (f64(r) if residual else 0)
    off = ref.product_bound(h, wdd) + off_h @ wdd.abs()
    within(y, y64, BF16 * y64.abs() + (1 + BF16) * off)

    dy = normal(6, rows, n, pitch=pitch and n + 40, shift=shift)
    g, u, dyd = kept_values(keep, "gate"), kept_values(keep, "up"), f64(dy)
    a, s = ref.act(g, act), ref.slope(g, act)
    dh = dyd @ wdd.T
    odh = ref.product_bound(dyd, wdd.T)
    dg, du, h = dh * u * s, dh * a, a * u
    fast = FAST * (1 + g.abs())
    odg = odh * (u * s).abs() + fast * (dh * u).abs() + BF16 * dg.abs() + 1e-30
    odu = odh * a.abs() + fast * dh.abs() + BF16 * du.abs() + 1e-30
    oh = fast * u.abs() + BF16 * h.abs() + 1e-30
    for dtype in (bf16, torch.float32):
        dx = torch.full((rows, n), float("nan"), dtype=bf16, device="cuda")
        grads = [torch.full(t.shape, float("nan"), dtype=dtype, device="cuda") for t in (wg, wu, wd)]
        binding.gated_ffn_grad(dy, x, wg, wu, wd, workspace=ws, activation=act, **keep, dx=dx, dw_gate=grads[0], dw_up=grads[1],
                               dw_down=grads[2], dx_addend=dy if residual else None)
        assert binding.layer_status(ws) == 0
        want = dg @ wgd.T + du @ wud.T + (dyd if residual else 0)
        off = odg @ wgd.abs().T + odu @ wud.abs().T + ref.product_bound(dg, wgd.T) + ref.product_bound(du, wud.T)
        off = off + (2 * -(-m // 16) * ref.ADD) * ((dg.abs() @ wgd.abs().T) + (du.abs() @ wud.abs().T))   # one chain for both
        within(dx, want, BF16 * want.abs() + (1 + BF16) * off)
        out = 0.0 if dtype == torch.float32 else BF16
        for got, left, right, off in ((grads[0], xd.T, dg, xd.abs().T @ odg), (grads[1], xd.T, du, xd.abs().T @ odu),
                                      (grads[2], h.T, dyd, oh.T @ dyd.abs())):
            want = left @ right
            within(got, want, out * want.abs() + (1 + out) * (off + 1.01 * ref.product_bound(left, right)) + 1e-30)


def test_gated_ffn_gradients_one_by_one():
    rows, n, m = 200, 64, 136
    x, dy = normal(1, rows, n), normal(2, rows, n)
    wg, wu, wd = normal(3, n, m, std=0.1), normal(4, n, m, std=0.1), normal(5, m, n, std=0.1)
    keep = {"gate": normal(6, rows, m), "up": normal(7, rows, m)}
    ws = workspace(binding.gated_ffn_grad_workspace_bytes(rows, n, m))
    whole = {"dx": torch.empty_like(x), "dw_gate": torch.empty_like(wg), "dw_up": torch.empty_like(wu), "dw_down": torch.empty_like(wd)}
    binding.gated_ffn_grad(dy, x, wg, wu, wd, workspace=ws, **keep, **whole)
    for names in (["dx"], ["dw_gate"], ["dw_up"], ["dw_down"], ["dw_up", "dw_down"], ["dx", "dw_gate", "dw_up"]):
        some = {k: torch.zeros_like(whole[k]) for k in names}
        needs_x = "dw_gate" in names or "dw_up" in names
        binding.gated_ffn_grad(dy, x if needs_x else None, wg, wu, wd, workspace=ws, **keep, **some)
        for k in names:
            want = f64(whole[k])
            # the reduction may be split differently: equal to two roundings
            assert ((f64(some[k]) - want).abs() <= 2 * BF16 * want.abs() + 1e-2 * BF16).all(), k


def test_gradients_against_differences():
    """The block's and the layer's gradients against differences of the 64-bit forward pass."""
    rows, n, m = 24, 16, 40
    x, wg, wu, wd, dy = (normal(i, *s, std=0.5) for i, s in enumerate([(rows, n), (n, m), (n, m), (m, n), (rows, n)]))
    gate, up = torch.empty(rows, m, dtype=bf16, device="cuda"), torch.empty(rows, m, dtype=bf16, device="cuda")
    ws = workspace(max(binding.gated_ffn_workspace_bytes(rows, n, m), binding.gated_ffn_grad_workspace_bytes(rows, n, m)))
    binding.gated_ffn(x, wg, wu, wd, torch.empty_like(x), ws, activation="gelu", gate=gate, up=up)
    got = {"x": torch.empty_like(x), "wg": torch.empty_like(wg), "wu": torch.empty_like(wu), "wd": torch.empty_like(wd)}
    binding.gated_ffn_grad(dy, x, wg, wu, wd, gate, up, ws, activation="gelu", dx=got["x"], dw_gate=got["wg"], dw_up=got["wu"], dw_down=got["wd"])
    v = {"x": f64(x), "wg": f64(wg), "wu": f64(wu), "wd": f64(wd)}
    loss = lambda v: float((((ref.act(v["x"] @ v["wg"], "gelu") * (v["x"] @ v["wu"])) @ v["wd"]) * f64(dy)).sum())  # noqa: E731
    g = torch.Generator().manual_seed(3)
    for name in v:
        d = torch.randn(v[name].shape, generator=g, dtype=torch.float64)
        e = 1e-5
        slope = (loss({**v, name: v[name] + e * d}) - loss({**v, name: v[name] - e * d})) / (2 * e)
        mine = float((f64(got[name]) * d).sum())
        # each element of the gradient carries at most four roundings of 2^-8 (gate, up, d_gate or h, itself), with signs of its own
        assert abs(mine - slope) <= 4 * BF16 * float((f64(got[name]) * d).norm()) * 3 + 1e-6 * abs(slope), name


@pytest.mark.parametrize("rows", [0, 1])
def test_no_rows_and_one(rows):
    n, m = 24, 40
    x, w, dy = normal(1, rows, n), normal(2, n, m), normal(3, rows, m)
    ws = workspace(1 << 20)
    y = torch.empty(rows, m, dtype=bf16, device="cuda")
    binding.linear(x, w, y, ws)
    dw, db = torch.full((n, m), 3.0, device="cuda"), torch.full((m,), 3.0, device="cuda")
    binding.linear_grad(dy, x, w, ws, dw=dw, dbias=db, dx=torch.empty_like(x))
    assert binding.layer_status(ws) == 0
    if rows == 0:
        assert (dw == 0).all() and (db == 0).all()
    wg, wu, wd = normal(4, n, m), normal(5, n, m), normal(6, m, n)
    gate, up = normal(7, rows, m), normal(8, rows, m)
    y, grads = torch.empty(rows, n, dtype=bf16, device="cuda"), [torch.full(s, 3.0, dtype=bf16, device="cuda") for s in ((n, m), (n, m), (m, n))]
    binding.gated_ffn(x, wg, wu, wd, y, ws)
    binding.gated_ffn_grad(normal(9, rows, n), x, wg, wu, wd, gate, up, ws, dw_gate=grads[0], dw_up=grads[1], dw_down=grads[2])
    assert binding.layer_status(ws) == 0
    if rows == 0:
        assert all((g == 0).all() for g in grads)


def test_what_is_not_finite_stays_in_its_row():
    rows, n, m = 300, 128, 256
    x, w = normal(1, rows, n), normal(2, n, m, std=0.1)
    ws = workspace(binding.linear_workspace_bytes(rows, n, m))
    clean, y = torch.empty(rows, m, dtype=bf16, device="cuda"), torch.empty(rows, m, dtype=bf16, device="cuda")
    keep = kept_buffers(rows, m, "e4m3", ["z"])
    binding.linear(x, w, clean, ws, activation="silu")
    x[5, 3], x[170, 0], x[299, 127] = float("nan"), float("inf"), float("-inf")
    binding.linear(x, w, y, ws, activation="silu", **keep)
    touched = torch.tensor([5, 170, 299], device="cuda")
    others = torch.ones(rows, dtype=torch.bool, device="cuda")
    others[touched] = False
    assert torch.equal(y[others], clean[others])
    assert y[5].isnan().all() and not y[170].isfinite().all() and not y[299].isfinite().all()
    assert keep["z"].float()[touched].isnan().all()
    assert not keep["z"].float()[others].isnan().any()


# ------------------------------------------------------------------------------------------------ streams, graphs, order
def test_same_bits_on_streams_and_in_replayed_graphs():
    rows, n, m = 700, 256, 512
    x, wg, wu, wd = normal(1, rows, n), normal(2, n, m, std=0.06), normal(3, n, m, std=0.06), normal(4, m, n, std=0.04)
    dy = normal(5, rows, n)

    def buffers():
        keep = kept_buffers(rows, m, "e4m3", ["gate", "up"])
        ws = workspace(max(binding.gated_ffn_workspace_bytes(rows, n, m), binding.gated_ffn_grad_workspace_bytes(rows, n, m)))
        out = {"y": torch.zeros_like(x), "dx": torch.zeros_like(x), "dw_gate": torch.zeros_like(wg), "dw_up": torch.zeros_like(wu),
               "dw_down": torch.zeros_like(wd)}
        return keep, ws, out

    def step(keep, ws, out):
        binding.gated_ffn(x, wg, wu, wd, out["y"], ws, residual=x, **keep)
        binding.gated_ffn_grad(dy, x, wg, wu, wd, workspace=ws, **keep, **{k: v for k, v in out.items() if k != "y"})

    first = buffers()
    step(*first)
    torch.cuda.synchronize()
    for _ in range(5):                                       # back to back on one workspace
        step(*first)
    second, third = buffers(), buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                            # two streams at once, a workspace each
        step(*second)
    step(*first)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(*third)
    for t in third[2].values():
        t.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for other in (second, third):
        assert binding.layer_status(other[1]) == 0
        for k, t in first[2].items():
            assert torch.equal(t, other[2][k]), k
    dy.mul_(2)                                               # a replay reads what its buffers hold then
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(third[2]["dw_down"].float(), 2 * first[2]["dw_down"].float())


def test_explicit_stream():
    rows, n, m = 64, 64, 64
    x, w = normal(1, rows, n), normal(2, n, m)
    y, z = torch.zeros(rows, m, dtype=bf16, device="cuda"), torch.zeros(rows, m, dtype=bf16, device="cuda")
    ws, other = workspace(binding.linear_workspace_bytes(rows, n, m)), workspace(binding.linear_workspace_bytes(rows, n, m))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    binding.linear(x, w, y, ws, stream=s)
    s.synchronize()
    binding.linear(x, w, z, other)
    assert torch.equal(y, z)


# ------------------------------------------------------------------------------------------------ checkpoints
@pytest.mark.parametrize("rows,n,pitch,shift", [(1, 1, 0, 0), (3, 31, 0, 0), (5, 32, 0, 0), (4, 33, 0, 0), (17, 64, 80, 8), (9, 100, 0, 0),
                                                (64, 1000, 0, 0), (33, 72, 99, 1), (1000, 256, 0, 0), (2, 40000, 0, 0)])
def test_checkpoint_pack_and_unpack(rows, n, pitch, shift):
    x = normal(1, rows, n, pitch=pitch, shift=shift)
    x.mul_(torch.exp(normal(2, n, std=3.0, dtype=torch.float32)).to(bf16))
    if rows > 2 and n > 8:
        x[1, :] = 0
        x[2, 3], x[2, 7], x[0, 5] = float("inf"), float("nan"), 2.0**-133
        x[0, n - 1] = 3.3e38
    codes = torch.zeros(rows, n, dtype=torch.uint8, device="cuda").view(e4m3)
    scale = torch.zeros(rows, binding.checkpoint_scales(n), dtype=torch.uint8, device="cuda").view(e8m0)
    binding.checkpoint_pack(x, codes, scale)
    want_codes, want_scale = ref.pack(x.float().cpu())
    assert torch.equal(scale.view(torch.uint8).cpu(), want_scale)
    nan = want_codes.float().isnan()
    assert torch.equal(codes.view(torch.uint8).cpu()[~nan], want_codes.view(torch.uint8)[~nan])
    assert codes.float().cpu()[nan].isnan().all()
    guard = torch.full((rows, n + 5), 7.0, dtype=bf16, device="cuda")
    out = guard[:, 2:n + 2] if pitch else guard[:, :n]
    binding.checkpoint_unpack(codes, scale, out)
    want = ref.unpack(want_codes, want_scale).float().to(bf16)
    assert torch.equal(out.cpu()[~nan], want[~nan]) and out.cpu()[nan].isnan().all()
    assert (guard[:, n + 2:] == 7).all()
    # every value that has a code comes back as itself
    again = torch.zeros_like(codes.view(torch.uint8)).view(e4m3)
    binding.checkpoint_pack(out, again, scale)
    back = torch.empty(rows, n, dtype=bf16, device="cuda")
    binding.checkpoint_unpack(again, scale, back)
    assert torch.equal(back.cpu()[~nan], want[~nan])


def test_checkpoint_scale_bytes_at_the_ends():
    codes = torch.full((1, 96), 0x38, dtype=torch.uint8, device="cuda").view(e4m3)         # 1.0
    scale = torch.tensor([[0, 255, 254]], dtype=torch.uint8, device="cuda").view(e8m0)
    out = torch.empty(1, 96, dtype=bf16, device="cuda")
    binding.checkpoint_unpack(codes, scale, out)
    v = out.float().cpu()[0]
    assert (v[:32] == 2.0**-127).all() and v[32:64].isnan().all() and (v[64:] == 2.0**127).all()


# ------------------------------------------------------------------------------------------------ embedding
@pytest.mark.parametrize("rows,vocab,n,pad,shift", [(1, 1, 1, 0, 0), (5, 3, 8, 0, 0), (100, 50, 33, 0, 0), (300, 1000, 64, 16, 8), (77, 7, 100, 3, 1),
                                                    (1000, 5000, 264, 0, 0), (40, 600, 2056, 0, 0)])
@pytest.mark.parametrize("table_dtype", [torch.float32, bf16])
@pytest.mark.parametrize("out_dtype", [torch.float32, bf16])
def test_embedding(rows, vocab, n, pad, shift, table_dtype, out_dtype):
    table = normal(1, vocab, n, dtype=table_dtype)
    tokens = torch.randint(-1, vocab + 1, (rows,), generator=gen(2), device="cuda", dtype=torch.int32)   # some outside the table
    tokens[0] = vocab - 1
    guard = torch.full((rows, n + pad + 8), 7.0, dtype=out_dtype, device="cuda")
    out = guard[:, shift:shift + n]
    binding.embedding(tokens, table, out, scale=3.5)
    t = tokens.cpu()
    live = (t >= 0) & (t < vocab)
    want = torch.where(live[:, None], table.float().cpu()[t.clamp(0, vocab - 1).long()] * 3.5, torch.zeros(())).to(out_dtype)
    assert torch.equal(out.cpu(), want)
    assert (guard[:, shift + n:] == 7).all()


GRADS = [  # rows, vocab, width, distribution of the tokens
    (1, 1, 1, "all"), (1, 300, 64, "all"), (200, 800, 64, "zipf"), (9, 5, 33, "all"), (500, 3, 40, "all"), (8192, 511, 72, "zipf"),
    (8192, 512, 8, "zipf"), (8193, 513, 16, "zipf"), (5000, 40000, 264, "zipf"), (20000, 3000, 136, "zipf"), (16385, 100, 24, "one"),
    (30000, 300000, 24, "all"), (1500, 400, 40, "zipf"), (257, 5000, 24, "zipf"), (256, 5000, 24, "zipf"), (70000, 300000, 8, "zipf"),
    (4097, 64, 2056, "zipf"), (3000, 70, 8, "outside"), (1100000, 1500, 8, "zipf"),
]


@pytest.mark.parametrize("rows,vocab,n,kind", GRADS)
def test_embedding_grad(rows, vocab, n, kind):
    u = torch.rand(rows, generator=gen(1), device="cuda", dtype=torch.float64)
    tokens = {"zipf": ((vocab + 1.0) ** u - 1).floor().clamp(0, vocab - 1), "all": torch.floor(u * (vocab + 2)) - 1,
              "one": torch.full_like(u, vocab - 1), "outside": torch.where(u < 0.5, -1.0, float(vocab))}[kind].to(torch.int32)
    ws = workspace(binding.embedding_grad_workspace_bytes(rows, vocab, n))
    t = tokens.long()
    at = torch.where((t >= 0) & (t < vocab), t, vocab)
    counts = torch.bincount(at, minlength=vocab + 1)[:vocab].cpu().double()
    for dy_dtype, out_dtype in ((bf16, torch.float32), (torch.float32, bf16)):
        dy = normal(2, rows, n, dtype=dy_dtype, pitch=n + 8, shift=0)
        exact = torch.zeros(vocab + 1, n, dtype=torch.float64, device="cuda").index_add_(0, at, dy.double())[:vocab].cpu() * 0.75
        size = torch.zeros(vocab + 1, n, dtype=torch.float64, device="cuda").index_add_(0, at, dy.double().abs())[:vocab].cpu() * 0.75
        out = torch.full((vocab, n), float("nan"), dtype=out_dtype, device="cuda")
        binding.embedding_grad(tokens, dy, out, ws, scale=0.75)
        rounding = 2.0**-24 if out_dtype == torch.float32 else BF16
        # a row of c tokens: c additions and the scale, each off by half a step of fp32
        bound = rounding * exact.abs() + (counts[:, None] + 2) * 2.0**-24 * size
        got = f64(out)
        assert ((got - exact).abs() <= bound).all()
        assert (got[counts == 0] == 0).all()
        again = torch.empty_like(out)
        binding.embedding_grad(tokens, dy, again, ws, scale=0.75)
        assert torch.equal(out, again)


def test_embedding_grad_against_the_loop():
    tokens = torch.tensor([3, -1, 0, 3, 9, 2, 3, 3], dtype=torch.int32, device="cuda")
    dy = normal(1, 8, 10, dtype=torch.float32)
    out = torch.empty(4, 10, device="cuda")
    binding.embedding_grad(tokens, dy, out, workspace(binding.embedding_grad_workspace_bytes(8, 4, 10)), scale=2.0)
    want = ref.embedding_grad(tokens, dy.cpu(), 4, 2.0)
    assert ((f64(out) - want).abs() <= 6 * 2.0**-24 * 8 * want.abs().clamp_min(1)).all()


def test_embedding_grad_without_rows_and_in_a_graph():
    out = torch.full((50, 16), 3.0, device="cuda")
    ws = workspace(binding.embedding_grad_workspace_bytes(20000, 50, 16))
    binding.embedding_grad(torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, 16, dtype=bf16, device="cuda"), out, ws)
    assert (out == 0).all()
    tokens = torch.randint(0, 50, (20000,), generator=gen(1), device="cuda", dtype=torch.int32)
    dy = normal(2, 20000, 16)
    binding.embedding_grad(tokens, dy, out, ws)
    eager = out.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        binding.embedding_grad(tokens, dy, out, ws)
    out.fill_(1)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, eager)
    tokens.fill_(7)                                          # other tokens, other runs
    graph.replay()
    torch.cuda.synchronize()
    assert (out[:7] == 0).all() and (out[8:] == 0).all()
    want = f64(dy).sum(0)
    assert ((f64(out)[7] - want).abs() <= 20002 * 2.0**-24 * f64(dy).abs().sum(0)).all()


def test_columns_of_one_tensor():
    """x, y, the residual, dy and dx as columns of one tensor: the columns between them stay."""
    rows, n, m = 150, 64, 72
    wide = normal(1, rows, n + 3 * m + n + 16)
    x, y, r, dy, dx = (wide[:, a:a + k] for a, k in ((0, n), (n, m), (n + m, m), (n + 2 * m, m), (n + 3 * m, n)))
    before = wide.clone()
    w = normal(2, n, m, std=0.1)
    ws = workspace(max(binding.linear_workspace_bytes(rows, n, m), binding.linear_grad_workspace_bytes(rows, n, m)))
    binding.linear(x, w, y, ws, residual=r, activation="gelu")
    binding.linear_grad(dy, x, w, ws, dx=dx)
    want_y, want_dx = torch.empty(rows, m, dtype=bf16, device="cuda"), torch.empty(rows, n, dtype=bf16, device="cuda")
    binding.linear(x.contiguous(), w, want_y, ws, residual=r.contiguous(), activation="gelu")
    binding.linear_grad(dy.contiguous(), None, w, ws, dx=want_dx)
    assert torch.equal(y, want_y) and torch.equal(dx, want_dx)
    before[:, n:n + m], before[:, n + 3 * m:n + 3 * m + n] = want_y, want_dx
    assert torch.equal(wide, before)


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_activations_far_out(act):
    """z = x w with a 1 x 1 weight of one: the activation of every kind of value."""
    v = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1e-40, 3.0, -3.0, 9.0, -9.0, 30.0, -30.0, 200.0, -200.0, 3e38, -3e38, float("inf"), float("nan")])
    x = v.to(bf16).cuda()[:, None].contiguous()
    y = torch.empty_like(x)
    ws = workspace(max(binding.linear_workspace_bytes(len(v), 1, 1), binding.linear_grad_workspace_bytes(len(v), 1, 1)))
    one = torch.ones(1, 1, dtype=bf16, device="cuda")
    z = torch.empty_like(x)
    binding.linear(x, one, y, ws, activation=act, z=z)
    xd = f64(x)[:, 0]
    want = ref.act(xd, act)
    got = f64(y)[:, 0]
    assert got[-1].isnan() and torch.isinf(got[-2]) and got[-2] > 0
    assert ((got - want).abs() <= BF16 * want.abs() + 2 * FAST * xd.abs().clamp(max=1) + 1e-37)[:-2].all()
    dx = torch.empty_like(x)
    binding.linear_grad(torch.ones_like(x), None, one, ws, z=z, activation=act, dx=dx)
    slope = ref.slope(xd, act)
    # dz is rounded to bf16, and again as dx
    assert ((f64(dx)[:, 0] - slope).abs() <= 2.01 * BF16 * slope.abs() + 4 * FAST)[:-2].all()


@pytest.mark.parametrize("rows,n,m,aligned", [(5, 16, 24, True), (130, 33, 70, False), (256, 2048, 1000, True), (40, 4096, 64, True),
                                              (3000, 64, 264, True), (333, 1001, 777, False)])
def test_nothing_is_written_behind_the_workspace(rows, n, m, aligned):
    def scratch(nbytes):
        whole = torch.full((nbytes + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        return whole[:nbytes], whole[nbytes:]

    x, w, dy = normal(1, rows, n), normal(2, n, m, std=0.05), normal(3, rows, m)
    z, y = torch.empty(rows, m, dtype=bf16, device="cuda"), torch.empty(rows, m, dtype=bf16, device="cuda")
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(m, dtype=bf16, device="cuda")
    ws, behind = scratch(binding.linear_workspace_bytes(rows, n, m, aligned))
    binding.linear(x, w, y, ws, activation="silu", z=z)
    assert (behind == 0xA5).all() and binding.layer_status(ws) == 0
    ws, behind = scratch(binding.linear_grad_workspace_bytes(rows, n, m, aligned))
    binding.linear_grad(dy, x, w, ws, z=z, activation="silu", dx=dx, dw=dw, dbias=db)
    assert (behind == 0xA5).all() and binding.layer_status(ws) == 0
    wd, yn = normal(4, m, n, std=0.05), torch.empty_like(x)
    ws, behind = scratch(binding.gated_ffn_workspace_bytes(rows, n, m, aligned))
    binding.gated_ffn(x, w, w, wd, yn, ws, gate=z, up=y)
    assert (behind == 0xA5).all() and binding.layer_status(ws) == 0
    ws, behind = scratch(binding.gated_ffn_grad_workspace_bytes(rows, n, m, aligned))
    binding.gated_ffn_grad(yn, x, w, w, wd, z, y, ws, dx=dx, dw_gate=dw, dw_up=torch.empty_like(w), dw_down=torch.empty_like(wd))
    assert (behind == 0xA5).all() and binding.layer_status(ws) == 0
    tokens = torch.randint(-1, m, (rows,), generator=gen(5), device="cuda", dtype=torch.int32)
    ws, behind = scratch(binding.embedding_grad_workspace_bytes(rows, m, n))
    table = torch.full((m + 1, n), 7.0, dtype=bf16, device="cuda")
    binding.embedding_grad(tokens, x, table[:m], ws)
    assert (behind == 0xA5).all() and (table[m] == 7).all()


def test_linear_gradients_against_differences():
    rows, n, m = 24, 16, 40
    x, w, dy = normal(1, rows, n, std=0.5), normal(2, n, m, std=0.5), normal(3, rows, m, std=0.5)
    b = normal(4, m, std=0.5)
    z, y = torch.empty(rows, m, dtype=bf16, device="cuda"), torch.empty(rows, m, dtype=bf16, device="cuda")
    ws = workspace(max(binding.linear_workspace_bytes(rows, n, m), binding.linear_grad_workspace_bytes(rows, n, m)))
    binding.linear(x, w, y, ws, bias=b, activation="silu", z=z)
    got = {"x": torch.empty_like(x), "w": torch.empty_like(w), "b": torch.empty_like(b)}
    binding.linear_grad(dy, x, w, ws, z=z, activation="silu", dx=got["x"], dw=got["w"], dbias=got["b"])
    v = {"x": f64(x), "w": f64(w), "b": f64(b)}
    loss = lambda v: float((ref.act(v["x"] @ v["w"] + v["b"], "silu") * f64(dy)).sum())  # noqa: E731
    g = torch.Generator().manual_seed(4)
    for name in v:
        d = torch.randn(v[name].shape, generator=g, dtype=torch.float64)
        e = 1e-5
        slope = (loss({**v, name: v[name] + e * d}) - loss({**v, name: v[name] - e * d})) / (2 * e)
        mine = float((f64(got[name]) * d).sum())
        # three roundings of 2^-8 an element (z, dz, itself), with signs of their own
        assert abs(mine - slope) <= 3 * BF16 * float((f64(got[name]) * d).norm()) * 3 + 1e-6 * abs(slope), name


def test_host_threads_with_streams_and_workspaces_of_their_own():
    import threading

    rows, n, m = 300, 128, 256
    w, wd = normal(1, n, m, std=0.1), normal(2, m, n, std=0.06)
    tokens = torch.randint(-1, 50, (rows,), generator=gen(3), device="cuda", dtype=torch.int32)
    inputs = [normal(10 + i, rows, n) for i in range(4)]

    def work(x, ws, out, keep):
        binding.gated_ffn(x, w, w, wd, out["y"], ws, residual=x, **keep)
        binding.gated_ffn_grad(out["y"], x, w, w, wd, workspace=ws, **keep, dx=out["dx"], dw_down=out["dw"])
        binding.embedding_grad(tokens, out["dx"], out["table"], ws)

    def buffers():
        size = max(binding.gated_ffn_workspace_bytes(rows, n, m), binding.gated_ffn_grad_workspace_bytes(rows, n, m),
                   binding.embedding_grad_workspace_bytes(rows, 50, n))
        out = {"y": torch.zeros(rows, n, dtype=bf16, device="cuda"), "dx": torch.zeros(rows, n, dtype=bf16, device="cuda"),
               "dw": torch.zeros(m, n, device="cuda"), "table": torch.zeros(50, n, device="cuda")}
        return workspace(size), out, kept_buffers(rows, m, "e4m3", ["gate", "up"])

    alone = [buffers() for _ in inputs]
    for x, b in zip(inputs, alone):
        work(x, *b)
    torch.cuda.synchronize()
    together, failed = [buffers() for _ in inputs], []

    def thread(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    work(inputs[i], *together[i])
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=thread, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed
    for a, b in zip(alone, together):
        for k in a[1]:
            assert torch.equal(a[1][k], b[1][k]), k
