"""The cases of the layers' GPU tests reach every kernel of the products, as the plan that the calls follow picks it."""
import ctypes

import pytest

import layers_cases as cases
from paper_2305_12213_b200 import binding
from paper_2305_12213_b200 import build as dbuild


@pytest.fixture(scope="module", autouse=True)
def lib():
    dbuild.build()
    return binding.lib()


def test_every_kernel_has_a_case():
    got = cases.plans(binding.bench_layer_plan)
    for product in cases.LINEAR_PRODUCTS + cases.GATED_PRODUCTS:
        for ctas, columns in cases.SHAPES:
            if product == "gated_h" and columns == 64:
                continue                                        # gate and up side by side need 128 columns
            for cut in (False, True):
                assert (product, ctas, columns, cut) in got, (product, ctas, columns, cut)


@pytest.mark.parametrize("product", cases.LINEAR_PRODUCTS + cases.GATED_PRODUCTS)
def test_pairs_have_remainders_odd_sizes_and_several_tiles(product):
    got = cases.plans(binding.bench_layer_plan)
    sizes = got[(product, 2, 256, False)] + got[(product, 2, 256, True)]
    assert any(n % 8 or m % 8 for _, n, m in sizes) and any(n % 8 == 0 and m % 8 == 0 for _, n, m in sizes)
    most = max(cases.tiles_a_worker(product, binding.bench_layer_plan(product, *s), *s) for s in sizes)
    assert most >= (2 if product.endswith("dw") else 3)


def test_plan_query_refusals(lib):
    out = (ctypes.c_int32 * 3)()
    at = ctypes.addressof(out)
    for bad in ((None, at, at), (at, None, at), (at, at, None)):
        assert lib.db_bench_layer_plan(0, 8, 8, 8, *bad) == binding.DB_ERR_NULL
    for bad in ((-1, 8, 8), (0, 8, 8), (8, 0, 8), (8, 8, 0), (2**30 + 1, 8, 8), (8, 2**24 + 1, 8)):
        assert lib.db_bench_layer_plan(0, *bad, at, at, at) == binding.DB_ERR_ARG
    assert lib.db_bench_layer_plan(8, 8, 8, 8, at, at, at) == lib.db_bench_layer_plan(-1, 8, 8, 8, at, at, at) == binding.DB_ERR_UNSUPPORTED
    assert binding.bench_layer_plan("linear_y", 1, 1, 1) == (1, 64, 1)
