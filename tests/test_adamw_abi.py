"""AdamW plans and the gradient-norm plan on the CPU: sizes, refusals (nothing reaches the GPU), and the reference
that the GPU tests use, checked against torch and against itself."""
import ctypes
import math
import re
import os

import numpy as np
import pytest
import torch

import adamw_reference as ref
from paper_2305_12213_b200 import binding
from paper_2305_12213_b200 import build as dbuild

E = binding
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    dbuild.build()
    return binding.lib()


def _ptrs(values):
    return (ctypes.c_void_p * len(values))(*values)


def _create(lib, **kw):
    """A call that is valid but for `kw`; pointers are far apart and never followed."""
    a = dict(K=2, T=2, sizes=[300, 2048], grads=[0x10000000 * (i + 1) for i in range(4)], params=[0x100000000, 0x110000000],
             copy=None, first=[0x120000000, 0x130000000], second=[0x140000000, 0x150000000], state=E.DB_F32, ms=None, us=None,
             wd=None, flags=0, grad=E.DB_F32, table=0x200000000, nbytes=None)
    a.update(kw)
    sizes = (ctypes.c_int64 * len(a["sizes"]))(*a["sizes"]) if a["sizes"] is not None else None
    table = lambda v: None if v is None else _ptrs(v)  # noqa: E731
    wd = None if a["wd"] is None else (ctypes.c_float * len(a["wd"]))(*a["wd"])
    nbytes = a["nbytes"]
    if nbytes is None:
        nbytes = 1 << 24
    out = ctypes.c_void_p(1)
    st = lib.db_adamw_plan_create(ctypes.byref(out), table(a["grads"]), a["grad"], a["K"], sizes, a["T"], table(a["params"]),
                                  table(a["copy"]), table(a["first"]), table(a["second"]), a["state"], table(a["ms"]),
                                  table(a["us"]), wd, a["flags"], a["table"], nbytes, None)
    assert st != E.DB_OK and not out.value
    return st


def test_constants_are_the_headers():
    text = open(os.path.join(ROOT, "include", "dynbatch.h")).read()
    assert int(re.search(r"#define\s+DB_ADAMW_BLOCK\s+(\d+)", text).group(1)) == E.DB_ADAMW_BLOCK == ref.BLOCK
    assert int(re.search(r"#define\s+DB_ADAMW_CLIP\s+(\d+)u", text).group(1)) == E.DB_ADAMW_CLIP
    assert int(re.search(r"DB_E4M3\s*=\s*(\d+)", text).group(1)) == E.DB_E4M3


def test_device_bytes(lib):
    def need(sizes, K=2, dt=E.DB_F32, flags=0, state=E.DB_F32):
        return lib.db_adamw_plan_device_bytes(K, dt, state, (ctypes.c_int64 * max(1, len(sizes)))(*sizes), len(sizes), flags)
    n = 100_000
    C = E.DB_ADAMW_CLIP
    assert need([n]) > 0 and need([n], flags=C) < need([n]) + 4 * n                      # 8 bytes of gradient: read twice
    assert need([n], K=3, flags=C) >= need([n], K=3) + 4 * n                              # more: staged
    assert need([n], K=4, dt=E.DB_BF16, flags=C) < need([n], K=4, dt=E.DB_BF16) + 4 * n
    assert need([n], state=E.DB_E4M3) > 0 and need([0, 0]) > 0
    assert need([n], K=0) == need([n], K=65) == need([-1]) == need([]) == need([n], dt=E.DB_E4M3) == need([n], flags=2) == 0
    assert need([n], state=E.DB_BF16) == 0
    assert need([2**63 - 1]) == 0 and need([2**62, 2**62, 2**62]) == 0                   # more steps than a grid has
    norm = lambda K, dt, s: lib.db_grad_norm_plan_device_bytes(K, dt, (ctypes.c_int64 * len(s))(*s), len(s))  # noqa: E731
    assert norm(1, E.DB_BF16, [1]) > 0 and norm(1, 7, [1]) == 0 and norm(1, E.DB_F32, [2**63 - 1]) == 0


def test_create_refusals(lib):
    assert _create(lib, grads=None) == E.DB_ERR_NULL
    assert _create(lib, params=None) == E.DB_ERR_NULL
    assert _create(lib, first=None) == E.DB_ERR_NULL
    assert _create(lib, second=None) == E.DB_ERR_NULL
    assert _create(lib, sizes=None) == E.DB_ERR_NULL
    assert _create(lib, table=None) == E.DB_ERR_NULL
    assert _create(lib, K=0) == E.DB_ERR_ARG
    assert _create(lib, K=65) == E.DB_ERR_ARG
    assert _create(lib, T=0) == E.DB_ERR_ARG
    assert _create(lib, sizes=[300, -1]) == E.DB_ERR_ARG
    assert _create(lib, sizes=[300, 2**63 - 1]) == E.DB_ERR_ARG
    assert _create(lib, flags=4) == E.DB_ERR_ARG
    assert _create(lib, grad=E.DB_E4M3) == E.DB_ERR_UNSUPPORTED
    assert _create(lib, state=E.DB_BF16) == E.DB_ERR_UNSUPPORTED
    assert _create(lib, state=E.DB_E4M3) == E.DB_ERR_NULL                               # no scales
    assert _create(lib, state=E.DB_E4M3, ms=[0x160000000, None], us=[0x170000000, 0x180000000]) == E.DB_ERR_NULL
    assert _create(lib, copy=[0x160000000, None]) == E.DB_ERR_NULL
    assert _create(lib, params=[0x100000000, None]) == E.DB_ERR_NULL
    assert _create(lib, grads=[0x10000000, 0x20000000, None, 0x40000000]) == E.DB_ERR_NULL
    assert _create(lib, params=[0x100000002, 0x110000000]) == E.DB_ERR_ARG              # off its element's alignment
    assert _create(lib, copy=[0x160000001, 0x170000000]) == E.DB_ERR_ARG
    assert _create(lib, grads=[0x10000001, 0x20000000, 0x30000000, 0x40000000], grad=E.DB_BF16) == E.DB_ERR_ARG
    assert _create(lib, wd=[0.1, float("nan")]) == E.DB_ERR_ARG
    assert _create(lib, table=0x200000010) == E.DB_ERR_ARG
    assert _create(lib, nbytes=256) == E.DB_ERR_ARG
    # overlaps: state with state, a gradient with a state, the table with a state, the same tensor twice
    assert _create(lib, first=[0x100000004, 0x130000000]) == E.DB_ERR_ARG
    assert _create(lib, params=[0x100000000, 0x100000000]) == E.DB_ERR_ARG
    assert _create(lib, grads=[0x10000000, 0x20000000, 0x100000000 + 4 * 299, 0x40000000]) == E.DB_ERR_ARG
    assert _create(lib, params=[0x200000000, 0x110000000]) == E.DB_ERR_ARG
    assert _create(lib, state=E.DB_E4M3, ms=[0x160000000, 0x170000000], us=[0x160000004, 0x180000000]) == E.DB_ERR_ARG


def test_norm_create_refusals(lib):
    def create(K=1, T=1, sizes=(300,), grads=(0x10000000,), dt=E.DB_F32, table=0x200000000, nbytes=1 << 20):
        out = ctypes.c_void_p(1)
        st = lib.db_grad_norm_plan_create(ctypes.byref(out), None if grads is None else _ptrs(grads), dt, K,
                                          (ctypes.c_int64 * len(sizes))(*sizes), T, table, nbytes, None)
        assert not out.value
        return st
    assert create(grads=None) == E.DB_ERR_NULL
    assert create(grads=(None,)) == E.DB_ERR_NULL
    assert create(table=None) == E.DB_ERR_NULL
    assert create(K=0) == create(K=65) == create(T=0) == create(sizes=(-5,)) == E.DB_ERR_ARG
    assert create(dt=E.DB_E4M3) == E.DB_ERR_UNSUPPORTED
    assert create(grads=(0x10000002,)) == E.DB_ERR_ARG
    assert create(nbytes=64) == create(table=0x200000001) == E.DB_ERR_ARG
    assert create(grads=(0x200000000,)) == E.DB_ERR_ARG                                  # a gradient inside the table


def test_null_plans(lib):
    b = (ctypes.c_int32 * 1)(1)
    assert lib.db_aggregate_adamw_multi(None, b, 0.1, 0.9, 0.9, 0.0, 1, 0.0, 0, None, None) == E.DB_ERR_NULL
    assert lib.db_grad_norm_multi(None, b, 0x1000, None) == E.DB_ERR_NULL
    assert lib.db_adamw_plan_destroy(None) == E.DB_OK and lib.db_grad_norm_plan_destroy(None) == E.DB_OK


def test_binding_refusals():
    g, p = [[torch.zeros(4)]], [torch.zeros(4)]
    with pytest.raises(TypeError):
        E.AdamWPlan(g, p, [torch.zeros(4)], [torch.zeros(4)])                            # not on a GPU
    with pytest.raises(TypeError):
        E.GradNormPlan(g)
    with pytest.raises(ValueError):
        E.AdamWPlan([], p, p, p)
    with pytest.raises(ValueError):
        E.AdamWPlan([[torch.zeros(4), torch.zeros(4)]], p, p, p)
    with pytest.raises(TypeError):
        E.GradNormPlan([[torch.zeros(4, dtype=torch.float16)]])


# ---- the reference itself ---------------------------------------------------------------------------
def test_reference_step_is_torch_adamw():
    rng = np.random.default_rng(3)
    p0 = rng.standard_normal(50)
    tp = torch.nn.Parameter(torch.tensor(p0))
    lr, b1, b2, eps, wd = (ref.f32(v) for v in (1e-2, 0.9, 0.999, 1e-8, 0.1))
    opt = torch.optim.AdamW([tp], lr=lr, betas=(b1, b2), eps=eps, weight_decay=wd)
    p, m, u = p0, np.zeros(50), np.zeros(50)
    for t in range(1, 6):
        g = rng.standard_normal(50).astype(np.float32)
        tp.grad = torch.tensor(g.astype(np.float64))
        opt.step()
        (p, m, u), _ = ref.step([g], [3], p, m, u, lr, b1, b2, eps, t, wd)
        assert np.abs(p - tp.detach().numpy()).max() < 1e-12


def test_reference_codes_are_torchs_e4m3():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.tensor(codes).view(torch.float8_e4m3fn).float().numpy()
    got = ref.e4m3_values(codes)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~np.isnan(got)], want[~np.isnan(want)])
    # without chance a value is cut to the code below it; with all of it, every value that is no code goes up
    v = np.sort(got[:127])
    y = np.random.default_rng(0).uniform(0, 448, 4000)
    below = v[np.searchsorted(v, y, side="right") - 1]
    assert np.array_equal(ref.round_up_by_chance(y, np.zeros(4000)), below)
    assert np.array_equal(ref.round_up_by_chance(v, np.full(127, 65535.0)), v)


def test_reference_rounding_is_unbiased_and_bits_are_even():
    """Mean of 2^20 rounded copies of y: the chance has 16 bits, so the mean may be off by q 2^-17 on the average plus
    five standard errors of at most q / 2 / 2^10."""
    n = 1 << 20
    for seed, step in ((0, 1), (123456789, 77), (2**63, 5)):
        r = ref.random_bits(np.arange(n) + (2**32 - n // 2), seed, step)
        for chance in (r & np.uint64(0xFFFF), r >> np.uint64(16)):
            chance = chance.astype(np.float64)
            for y in (0.0011, 0.7, 100.3, 447.9):
                q = 2.0 ** (max(math.floor(math.log2(y)), -6) - 3)
                mean = ref.round_up_by_chance(np.full(n, y), chance).mean()
                assert abs(mean - y) <= q * (2.0**-16 + 5 * 0.5 / 2**10)
