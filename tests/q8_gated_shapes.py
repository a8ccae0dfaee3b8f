"""The shapes at which the products of 8-bit integers and the gated projection are tested, chosen so that every kernel takes some of them, with
ragged edges and without."""
from __future__ import annotations

KERNELS = ("waves32", "waves32_wide", "waves64", "square128", "square256")

# m, n, k of fh_q8_matmul
PRODUCTS = [(1, 1, 1), (1, 16, 128), (1, 4096, 4096), (3, 1000, 8192), (5, 100, 40), (16, 2000, 1500), (17, 33, 129), (31, 64, 4096), (64, 64, 64), (65, 130, 257),
            (197, 1000, 1537), (256, 256, 256), (300, 513, 4100), (1000, 768, 2048), (513, 2049, 640), (8192, 24, 100), (4100, 1030, 96), (2048, 2304, 768), (3684, 3472, 17),
            (4353, 2305, 640)]
# m, n, k of fh_q8_gated
GATED = [(1, 1, 1), (1, 4096, 4096), (2, 100, 300), (7, 1000, 512), (9, 25, 4087), (16, 515, 2000), (33, 17, 129), (64, 64, 128), (65, 130, 257), (200, 768, 768),
         (292, 1638, 543), (509, 2731, 1023), (1000, 2048, 768), (4100, 300, 96), (3000, 1500, 640), (4003, 1568, 16)]
# tokens, features, hidden of the dense projection and its backward pass
DENSE = [(1, 1, 1), (1, 64, 64), (1, 4096, 1000), (2, 100, 30), (5, 515, 77), (16, 768, 2048), (17, 33, 65), (31, 128, 64), (64, 64, 32), (65, 130, 257), (200, 1000, 513),
         (333, 515, 1001), (256, 256, 128), (1025, 96, 40), (3000, 64, 300), (2048, 768, 1024), (4096, 520, 1300), (8200, 48, 40), (40, 2000, 1500)]
# the larger ones, one activation each: (dtype, tokens, features, hidden)
LARGE = [("bf16", 9731, 261, 636), ("bf16", 10542, 1229, 18), ("bf16", 10542, 1229, 26), ("bf16", 1, 3621, 1772), ("bf16", 11464, 3640, 26), ("bf16", 10707, 392, 2382),
         ("bf16", 8192, 768, 2048), ("f32", 10120, 968, 70), ("f32", 8130, 1025, 961), ("f32", 10701, 1466, 898)]
# rows that are apart by multiples of 16 bytes, none of them of 128: tokens, features, hidden, and how much wider the rows are
STRIDED = [(2048, 128, 1024, 8), (2100, 200, 1100, 24), (4200, 72, 1000, 40), (1500, 1000, 300, 16), (1030, 24, 2000, 4)]

# tokens, features, hidden of backward passes in bf16 that keep the rests of a rounding: up to 2^19 gradients of the gates, 2^27 products
WITH_RESTS = [(1, 1, 1), (1, 64, 64), (1, 4096, 1000), (2, 100, 30), (5, 515, 77), (17, 33, 65), (26, 63, 49), (64, 64, 32), (65, 130, 257), (200, 1000, 513), (333, 515, 700),
              (256, 256, 1024), (4096, 96, 64), (8192, 48, 32), (477, 20, 71), (15, 2100, 4100), (40, 2000, 1500),
              (500, 520, 500), (16, 4000, 2048), (8000, 900, 18), (8192, 540, 30)]


def products_of(dtype, tokens, features, hidden):
    """(m, n, chunks, fp32, may be shared, with rests) of the backward pass's products: both projections, dx, dW."""
    unit = 32 if dtype == "f32" else 64
    slow, padded = int(dtype == "f32"), -(-hidden // unit) * unit
    rests = int(not slow and tokens * hidden <= 2 ** 19 and tokens * hidden * features <= 2 ** 27)
    return {"pair": (tokens, 2 * hidden, -(-features // unit), slow, 0, rests), "dx": (tokens, features, (2 + 2 * rests) * padded // unit, slow, 0, rests),
            "dw": (padded + hidden, features, (1 + rests) * -(-tokens // unit), slow, 1, rests)}
