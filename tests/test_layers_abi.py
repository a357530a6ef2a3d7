"""Layers, checkpoints and embedding on the CPU: workspace sizes, refusals (nothing reaches the GPU), the binding's checks,
and the reference of the GPU tests checked against torch and against differences."""
import os
import re

import pytest
import torch

import layers_reference as ref
from paper_2305_12213_b200 import binding
from paper_2305_12213_b200 import build as dbuild

E = binding
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    dbuild.build()
    return binding.lib()


_A = [0x7000000000 + 0x100000000 * i for i in range(24)]      # addresses far apart, never followed


def _linear(lib, **kw):
    a = dict(x=_A[0], xp=64, w=_A[1], bias=_A[2], r=_A[3], rp=128, act=3, rows=100, n=64, m=128, y=_A[4], yp=128, z=_A[5],
             zs=_A[6], zt=E.DB_E4M3, ws=_A[7], nbytes=1 << 26)
    a.update(kw)
    return lib.db_linear(a["x"], a["xp"], a["w"], a["bias"], a["r"], a["rp"], a["act"], a["rows"], a["n"], a["m"], a["y"],
                         a["yp"], a["z"], a["zs"], a["zt"], a["ws"], a["nbytes"], None)


def _linear_grad(lib, **kw):
    a = dict(dy=_A[0], dyp=128, x=_A[1], xp=64, w=_A[2], z=_A[3], zs=_A[4], zt=E.DB_E4M3, act=3, rows=100, n=64, m=128,
             dx=_A[5], dxp=64, add=_A[6], addp=64, dw=_A[7], db=_A[8], gt=E.DB_BF16, ws=_A[9], nbytes=1 << 26)
    a.update(kw)
    return lib.db_linear_grad(a["dy"], a["dyp"], a["x"], a["xp"], a["w"], a["z"], a["zs"], a["zt"], a["act"], a["rows"],
                              a["n"], a["m"], a["dx"], a["dxp"], a["add"], a["addp"], a["dw"], a["db"], a["gt"], a["ws"],
                              a["nbytes"], None)


def _ffn(lib, **kw):
    a = dict(x=_A[0], xp=64, wg=_A[1], wu=_A[2], wd=_A[3], r=_A[4], rp=64, act=3, rows=100, n=64, m=256, y=_A[5], yp=64,
             g=_A[6], u=_A[7], gs=_A[8], us=_A[9], kt=E.DB_E4M3, ws=_A[10], nbytes=1 << 26)
    a.update(kw)
    return lib.db_gated_ffn(a["x"], a["xp"], a["wg"], a["wu"], a["wd"], a["r"], a["rp"], a["act"], a["rows"], a["n"], a["m"],
                            a["y"], a["yp"], a["g"], a["u"], a["gs"], a["us"], a["kt"], a["ws"], a["nbytes"], None)


def _ffn_grad(lib, **kw):
    a = dict(dy=_A[0], dyp=64, x=_A[1], xp=64, wg=_A[2], wu=_A[3], wd=_A[4], g=_A[5], u=_A[6], gs=_A[7], us=_A[8],
             kt=E.DB_E4M3, act=3, rows=100, n=64, m=256, dx=_A[9], dxp=64, add=_A[10], addp=64, dg=_A[11], du=_A[12],
             dd=_A[13], gt=E.DB_F32, ws=_A[14], nbytes=1 << 26)
    a.update(kw)
    return lib.db_gated_ffn_grad(a["dy"], a["dyp"], a["x"], a["xp"], a["wg"], a["wu"], a["wd"], a["g"], a["u"], a["gs"],
                                 a["us"], a["kt"], a["act"], a["rows"], a["n"], a["m"], a["dx"], a["dxp"], a["add"],
                                 a["addp"], a["dg"], a["du"], a["dd"], a["gt"], a["ws"], a["nbytes"], None)


def _embedding(lib, **kw):
    a = dict(t=_A[0], table=_A[1], tt=E.DB_BF16, rows=10, v=100, n=64, out=_A[2], op=64, ot=E.DB_F32)
    a.update(kw)
    return lib.db_embedding(a["t"], a["table"], a["tt"], 1.0, a["rows"], a["v"], a["n"], a["out"], a["op"], a["ot"], None)


def _embedding_grad(lib, **kw):
    a = dict(t=_A[0], dy=_A[1], dp=64, dt=E.DB_BF16, rows=10, v=100, n=64, out=_A[2], ot=E.DB_F32, ws=_A[3], nbytes=1 << 24)
    a.update(kw)
    return lib.db_embedding_grad(a["t"], a["dy"], a["dp"], a["dt"], 1.0, a["rows"], a["v"], a["n"], a["out"], a["ot"],
                                 a["ws"], a["nbytes"], None)


def _pack(lib, **kw):
    a = dict(x=_A[0], xp=64, rows=10, n=64, c=_A[1], s=_A[2])
    a.update(kw)
    return lib.db_checkpoint_pack(a["x"], a["xp"], a["rows"], a["n"], a["c"], a["s"], None)


def _unpack(lib, **kw):
    a = dict(x=_A[0], xp=64, rows=10, n=64, c=_A[1], s=_A[2])
    a.update(kw)
    return lib.db_checkpoint_unpack(a["c"], a["s"], a["rows"], a["n"], a["x"], a["xp"], None)


def test_constants_are_the_headers():
    text = open(os.path.join(ROOT, "include", "dynbatch.h")).read()
    for name, value in E.DB_ACTIVATIONS.items():
        assert int(re.search(r"DB_ACT_%s\s*=\s*(\d+)" % name.upper(), text).group(1)) == value
    assert int(re.search(r"#define\s+DB_CHECKPOINT_GROUP\s+(\d+)", text).group(1)) == E.DB_CHECKPOINT_GROUP == ref.GROUP


def test_workspace_bytes(lib):
    for f in (lib.db_linear_workspace_bytes, lib.db_linear_grad_workspace_bytes, lib.db_gated_ffn_workspace_bytes,
              lib.db_gated_ffn_grad_workspace_bytes):
        assert f(1, 1, 1, 1) > 0 and f(0, 8, 8, 1) > 0
        assert f(-1, 8, 8, 1) == f(8, 0, 8, 1) == f(8, 8, 0, 1) == f(2**30 + 1, 8, 8, 1) == f(8, 2**24 + 1, 8, 1) == 0
        assert f(2**30, 2**11, 8, 1) == 0 and f(8, 2**24, 2**24, 1) == 0           # more than 2^40 elements
        assert f(1000, 512, 2048, 0) > f(1000, 512, 2048, 1)
        assert f(1000, 511, 2048, 1) == f(1000, 511, 2048, 0)                      # odd features lie on no grid
    # the intermediate activations of the block: h forward, h, d_gate and d_up backward
    t, n, m = 4096, 512, 2048
    assert lib.db_gated_ffn_workspace_bytes(t, n, m, 1) >= 2 * t * m
    assert lib.db_gated_ffn_grad_workspace_bytes(t, n, m, 1) >= 6 * t * m
    g = lib.db_embedding_grad_workspace_bytes
    assert g(0, 1, 1) > 0 and g(1000, 50, 64) > 8 * 1000
    assert g(-1, 1, 1) == g(2**28 + 1, 1, 1) == g(1, 0, 1) == g(1, 2**26 + 1, 1) == g(1, 1, 0) == g(1, 1, 2**20 + 1) == 0


def test_linear_refusals(lib):
    for name in ("x", "w", "y", "ws"):
        assert _linear(lib, **{name: None}) == E.DB_ERR_NULL, name
    assert _linear(lib, zs=None) == E.DB_ERR_NULL
    for bad in (dict(rows=-1), dict(n=0), dict(m=0), dict(xp=63), dict(yp=127), dict(rp=127), dict(xp=2**31 + 1),
                dict(nbytes=lib.db_linear_workspace_bytes(100, 64, 128, 1) - 1), dict(ws=_A[7] + 16),
                dict(x=_A[0] + 1), dict(w=_A[1] + 1), dict(y=_A[4] + 1), dict(bias=_A[2] + 1), dict(r=_A[3] + 1),
                dict(y=_A[0] + 2 * 64 * 99), dict(y=_A[1]), dict(z=_A[4] + 2), dict(r=_A[4] + 256), dict(r=_A[4], rp=256),
                dict(zs=_A[5]), dict(y=_A[7] + 256), dict(z=_A[5] + 1, zt=E.DB_BF16),
                # an operand off the 16-byte grid needs the larger workspace
                dict(x=_A[0] + 2, nbytes=lib.db_linear_workspace_bytes(100, 64, 128, 0) - 1),
                dict(xp=65, nbytes=lib.db_linear_workspace_bytes(100, 64, 128, 0) - 1)):
        assert _linear(lib, **bad) == E.DB_ERR_ARG, bad
    for bad in (dict(act=4), dict(act=-1), dict(zt=E.DB_F32), dict(zt=7)):
        assert _linear(lib, **bad) == E.DB_ERR_UNSUPPORTED, bad


def test_columns_of_one_tensor_overlap_where_they_do(lib):
    wide = _A[0]
    apart = dict(x=wide, xp=400, y=wide + 2 * 64, yp=400, r=wide + 2 * 192, rp=400)
    for bad in (dict(y=wide + 2 * 63), dict(y=wide + 2 * 65), dict(r=wide + 2 * 191), dict(yp=336), dict(y=wide + 2 * 300),
                dict(y=wide + 2 * (400 * 99 - 64))):
        assert _linear(lib, **{**apart, **bad}) == E.DB_ERR_ARG, bad


def test_linear_grad_refusals(lib):
    for bad in (dict(dy=None), dict(x=None), dict(w=None), dict(z=None), dict(zs=None), dict(ws=None),
                dict(dx=None, add=None, dw=None, db=None)):
        assert _linear_grad(lib, **bad) == E.DB_ERR_NULL, bad
    for bad in (dict(rows=-1), dict(n=0), dict(m=2**24 + 1), dict(dyp=127), dict(xp=63), dict(dxp=63), dict(addp=63),
                dict(dx=None), dict(nbytes=lib.db_linear_grad_workspace_bytes(100, 64, 128, 1) - 1), dict(ws=_A[9] + 128),
                dict(dy=_A[0] + 1), dict(dw=_A[7] + 1), dict(db=_A[8] + 2, gt=E.DB_F32), dict(dw=_A[2]), dict(dx=_A[0]),
                dict(db=_A[7] + 64 * 128 * 2 - 2), dict(add=_A[5] + 2), dict(add=_A[5], addp=65), dict(dx=_A[4] + 2)):
        assert _linear_grad(lib, **bad) == E.DB_ERR_ARG, bad
    for bad in (dict(act=9), dict(gt=E.DB_E4M3), dict(zt=E.DB_F32)):
        assert _linear_grad(lib, **bad) == E.DB_ERR_UNSUPPORTED, bad


def test_gated_refusals(lib):
    for bad in (dict(x=None), dict(wg=None), dict(wu=None), dict(wd=None), dict(y=None), dict(ws=None), dict(g=None),
                dict(u=None), dict(gs=None), dict(us=None)):
        assert _ffn(lib, **bad) == E.DB_ERR_NULL, bad
    for bad in (dict(rows=-5), dict(n=0), dict(m=0), dict(xp=1), dict(yp=63), dict(rp=3),
                dict(nbytes=lib.db_gated_ffn_workspace_bytes(100, 64, 256, 1) - 1), dict(ws=_A[10] + 8), dict(u=_A[6] + 5),
                dict(y=_A[0]), dict(g=_A[5] + 1, kt=E.DB_BF16), dict(us=_A[8]), dict(wd=_A[3] + 1)):
        assert _ffn(lib, **bad) == E.DB_ERR_ARG, bad
    assert _ffn(lib, act=4) == _ffn(lib, kt=E.DB_F32) == E.DB_ERR_UNSUPPORTED


def test_gated_grad_refusals(lib):
    for bad in (dict(dy=None), dict(x=None), dict(wg=None), dict(wu=None), dict(wd=None), dict(g=None), dict(u=None),
                dict(gs=None), dict(us=None), dict(ws=None), dict(dx=None, add=None, dg=None, du=None, dd=None)):
        assert _ffn_grad(lib, **bad) == E.DB_ERR_NULL, bad
    for bad in (dict(rows=2**30 + 1), dict(dyp=63), dict(xp=63), dict(dxp=63), dict(addp=63), dict(dx=None),
                dict(nbytes=lib.db_gated_ffn_grad_workspace_bytes(100, 64, 256, 1) - 1), dict(ws=_A[14] + 255),
                dict(dg=_A[11] + 2), dict(du=_A[11]), dict(dd=_A[4]), dict(dx=_A[0]), dict(dx=_A[1]), dict(add=_A[9] + 4),
                dict(g=_A[5] + 1, kt=E.DB_BF16)):
        assert _ffn_grad(lib, **bad) == E.DB_ERR_ARG, bad
    for bad in (dict(act=-1), dict(gt=E.DB_E4M3), dict(kt=E.DB_F32)):
        assert _ffn_grad(lib, **bad) == E.DB_ERR_UNSUPPORTED, bad


def test_checkpoint_refusals(lib):
    for f in (_pack, _unpack):
        for name in ("x", "c", "s"):
            assert f(lib, **{name: None}) == E.DB_ERR_NULL
            assert f(lib, rows=0, **{name: None}) == E.DB_OK
        for bad in (dict(rows=-1), dict(n=0), dict(n=2**24 + 1), dict(xp=63), dict(x=_A[0] + 1), dict(c=_A[0]),
                    dict(s=_A[0] + 2 * 640 - 1), dict(rows=2**38, n=8), dict(rows=2**38 + 1, n=1)):
            assert f(lib, **bad) == E.DB_ERR_ARG, bad
    assert _pack(lib, s=_A[1] + 639) == E.DB_ERR_ARG


def test_embedding_refusals(lib):
    for name in ("t", "table", "out"):
        assert _embedding(lib, **{name: None}) == E.DB_ERR_NULL
    assert _embedding(lib, rows=0) == E.DB_OK
    for bad in (dict(rows=-1), dict(v=0), dict(n=0), dict(op=63), dict(t=_A[0] + 2), dict(table=_A[1] + 1), dict(out=_A[2] + 2),
                dict(out=_A[0]), dict(out=_A[1] + 64), dict(rows=2**28 + 1)):
        assert _embedding(lib, **bad) == E.DB_ERR_ARG, bad
    assert _embedding(lib, tt=E.DB_E4M3) == _embedding(lib, ot=5) == E.DB_ERR_UNSUPPORTED
    for name in ("t", "dy", "out", "ws"):
        assert _embedding_grad(lib, **{name: None}) == E.DB_ERR_NULL
    for bad in (dict(rows=-1), dict(v=0), dict(n=0), dict(dp=63), dict(t=_A[0] + 1), dict(dy=_A[1] + 1), dict(out=_A[2] + 2),
                dict(out=_A[1]), dict(ws=_A[3] + 64), dict(ws=_A[2] + 256), dict(v=2**26 + 1),
                dict(nbytes=lib.db_embedding_grad_workspace_bytes(10, 100, 64) - 1)):
        assert _embedding_grad(lib, **bad) == E.DB_ERR_ARG, bad
    assert _embedding_grad(lib, dt=E.DB_E4M3) == _embedding_grad(lib, ot=9) == E.DB_ERR_UNSUPPORTED


def test_binding_refuses_cpu_tensors_and_unknown_names():
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    w = torch.zeros(8, 8, dtype=torch.bfloat16)
    tokens = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: binding.linear(x, w, x.clone(), ws), lambda: binding.linear_grad(x, x, w, ws, dx=x.clone()),
                 lambda: binding.gated_ffn(x, w, w, w, x.clone(), ws),
                 lambda: binding.gated_ffn_grad(x, x, w, w, w, x, x, ws, dx=x.clone()),
                 lambda: binding.checkpoint_pack(x, x, x), lambda: binding.embedding(tokens, w, x),
                 lambda: binding.embedding_grad(tokens, x, w, ws)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        binding._activation("tanh")
    assert binding.checkpoint_scales(1) == 1 and binding.checkpoint_scales(33) == 2


# ------------------------------------------------------------------------------------------------ the reference itself
@pytest.mark.parametrize("name", ["none", "relu", "gelu", "silu"])
def test_reference_activations(name):
    z = torch.tensor([-30.0, -3.0, -0.5, 0.0, 1e-3, 0.7, 4.0, 30.0], dtype=torch.float64)
    stock = {"none": lambda v: v, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[name]
    assert torch.allclose(ref.act(z, name), stock(z), rtol=1e-12, atol=1e-300)
    z.requires_grad_()
    stock(z).sum().backward()
    assert torch.allclose(ref.slope(z.detach(), name), z.grad, rtol=1e-12, atol=1e-15)
    if name != "relu":
        d = 1e-6
        v = z.detach()
        assert torch.allclose(ref.slope(v, name), (ref.act(v + d, name) - ref.act(v - d, name)) / (2 * d), atol=1e-8)


def test_reference_pack():
    x = torch.zeros(1, 40)
    x[0, 0], x[0, 1], x[0, 2], x[0, 33] = 448.0, 1.0, 17.0, -1e-3
    codes, scale = ref.pack(x)
    assert scale.tolist() == [[127, 127 + math_power(1e-3)]]
    assert codes.float()[0, :3].tolist() == [448.0, 1.0, 16.0]                  # 17 lies between 16 and 18: to even
    x[0, 0] = 449.0
    codes, scale = ref.pack(x)
    assert scale[0, 0] == 128 and codes.float()[0, 0] == 224.0                  # 224.5 rounds to 224
    assert ref.pack(torch.zeros(2, 3))[1].tolist() == [[0], [0]]
    x[0, 5], x[0, 6] = float("inf"), float("nan")
    codes, scale = ref.pack(x)
    assert scale[0, 0] == 128 and codes.float()[0, 5:7].isnan().all()
    # values come back within half a step
    v = torch.randn(7, 100, generator=torch.Generator().manual_seed(1)) * torch.logspace(-12, 12, 100)
    codes, scale = ref.pack(v)
    step = torch.exp2(scale.double() - 127).repeat_interleave(32, 1)[:, :100]
    assert ((ref.unpack(codes, scale) - v.double()).abs() <= torch.maximum(2.0**-4 * v.double().abs(), 2.0**-10 * step)).all()


def math_power(x):
    """The smallest e with x <= 448 * 2^e."""
    e = -127
    while x > 448 * 2.0**e:
        e += 1
    return e


def test_reference_embedding():
    tokens = torch.tensor([3, -1, 0, 3, 9, 2], dtype=torch.int32)
    dy = torch.arange(12.0).view(6, 2)
    table = torch.zeros(4, 2, dtype=torch.float64, requires_grad=True)
    live = torch.tensor([0, 2, 3, 5])
    (torch.nn.functional.embedding(tokens[live].long(), table) * 2 * dy[live].double()).sum().backward()
    assert torch.equal(ref.embedding_grad(tokens, dy, 4, 2.0), table.grad)
