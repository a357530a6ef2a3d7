"""Sizes at which the plan picks every kernel of the layers' products: each tile shape, with the reduction whole and cut, for each
product, with row and column remainders; pairs of CTAs also off the 16-byte grid and with several tiles one after the other."""

LINEAR = [  # rows, n_in, n_out, bias, residual, activation, kept, pitch, shift
    (1, 4400, 1032, True, True, "none", "bf16", 0, 0),
    (1, 5920, 1992, True, False, "gelu", "e4m3", 0, 0),
    (2343, 8, 2143, False, True, "silu", "bf16", 0, 0),
    (10479, 9, 4128, True, True, "none", "none", 0, 0),
    (9236, 132, 1082, True, True, "gelu", "e4m3", 0, 0),
    (150, 5536, 1704, True, True, "relu", "bf16", 5552, 8),
    (11046, 4030, 8, False, True, "silu", "e4m3", 0, 0),
    (145, 3440, 4192, True, True, "gelu", "bf16", 0, 0),
    (8226, 1416, 8, True, False, "none", "bf16", 1424, 8),
    (4415, 8, 2992, False, True, "silu", "bf16", 0, 0),
    (2095, 2200, 8, True, True, "relu", "e4m3", 0, 0),
    (4643, 1315, 397, True, True, "silu", "bf16", 0, 0),
    (129, 1568, 4603, True, True, "gelu", "e4m3", 0, 0),
    (2050, 1096, 2184, True, True, "silu", "e4m3", 1112, 5),    # x copied onto the grid, the weights not
    (3000, 1032, 1544, True, True, "gelu", "bf16", 1048, 8),
    (8200, 264, 1544, False, True, "none", "none", 0, 0),
    (515, 96, 32000, True, False, "none", "none", 0, 0),        # a vocabulary's columns
    (70, 72, 32001, False, True, "gelu", "e4m3", 0, 0),
]
FFN = [  # rows, width, hidden, residual, activation, kept, pitch, shift
    (5016, 920, 9, True, "silu", "bf16", 0, 0),
    (1, 3385, 4104, True, "gelu", "e4m3", 0, 0),
    (2811, 4608, 16, False, "silu", "e4m3", 4616, 8),
    (5435, 8, 4128, True, "silu", "bf16", 0, 0),
    (1, 1048, 5264, False, "gelu", "bf16", 0, 0),
    (10851, 4200, 11, True, "silu", "e4m3", 0, 0),
    (7251, 136, 952, True, "gelu", "bf16", 144, 8),
    (409, 689, 2842, True, "silu", "bf16", 0, 0),
    (162, 2800, 2872, True, "gelu", "e4m3", 0, 0),
    (8607, 9, 5813, True, "silu", "e4m3", 0, 0),
    (3731, 200, 616, False, "relu", "bf16", 0, 0),
    (4363, 264, 1106, True, "silu", "bf16", 0, 0),
    (1, 408, 3338, True, "silu", "e4m3", 0, 0),
    (131, 4248, 2512, True, "silu", "bf16", 0, 0),
    (8804, 528, 144, True, "gelu", "e4m3", 0, 0),
    (1597, 2892, 264, True, "none", "bf16", 2900, 3),
    (145, 2407, 4264, True, "gelu", "bf16", 0, 0),
    (256, 2048, 1000, True, "silu", "e4m3", 0, 0),
    (2050, 1096, 2184, True, "gelu", "e4m3", 0, 0),
    (3000, 1032, 1544, False, "silu", "bf16", 1048, 8),
    (8200, 264, 1544, True, "silu", "e4m3", 0, 0),              # pairs with three tiles each
]

LINEAR_PRODUCTS, GATED_PRODUCTS = ("linear_y", "linear_dx", "linear_dw"), ("gated_h", "gated_y", "gated_dh", "gated_dx", "gated_dw")
SHAPES = ((2, 256), (2, 128), (1, 128), (1, 64))                # CTAs that share a tile, its columns


def plans(bench_layer_plan):
    """{(product, CTAs, columns, cut): [(rows, n_in, n_out)]} of all cases."""
    got = {}
    for cases, products in ((LINEAR, LINEAR_PRODUCTS), (FFN, GATED_PRODUCTS)):
        for rows, n, m, *_ in cases:
            for p in products:
                ctas, columns, pieces = bench_layer_plan(p, rows, n, m)
                got.setdefault((p, ctas, columns, pieces > 1), []).append((rows, n, m))
    return got


def tiles_a_worker(product, plan, rows, n, m):
    """Tiles that the busiest CTA, or pair, of 148 SMs computes one after the other."""
    ctas, columns, pieces = plan
    if product == "gated_h":
        columns //= 2
    out = {"linear_y": [(rows, m)], "linear_dx": [(rows, n)], "linear_dw": [(n, m)], "gated_h": [(rows, m)], "gated_y": [(rows, n)],
           "gated_dh": [(rows, m)], "gated_dx": [(rows, n)], "gated_dw": [(n, m), (n, m), (m, n)]}[product]
    tiles = pieces * sum(-(-a // (128 * ctas)) * -(-b // columns) for a, b in out)
    return -(-tiles // (74 if ctas == 2 else 296))
