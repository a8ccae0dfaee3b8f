"""Products of ragged sizes for every kernel of fh_mx_matmul: (kernel, m, n, k).  Which kernel a product takes is asserted on the host, and each
is compared with binary64 on the GPU, so that a rule that moves a shape to another kernel takes no kernel's test away unnoticed."""

KERNELS = ("waves32", "waves32_wide", "waves64", "square128", "square256")
SPLIT, RUNS, ORDER = "split", "runs", "order"          # a sum in parts; tiles of 64 in runs and in their order

PRODUCTS = [
    ("waves32", None, 640, 500, 8200),
    ("waves32", None, 900, 700, 3000),
    ("waves32", None, 1, 70000, 100),
    ("waves32_wide", None, 300, 333, 5000),
    ("waves32_wide", SPLIT, 96, 97, 40000),
    ("waves32_wide", SPLIT, 1, 33, 8200),
    ("waves64", RUNS, 2300, 770, 8200),
    ("waves64", RUNS, 770, 777, 8200),
    ("waves64", RUNS, 450, 4000, 2050),
    ("waves64", ORDER, 1000, 1000, 2000),
    ("waves64", ORDER, 700, 1100, 4100),
    ("waves64", ORDER, 500, 2000, 4090),
    ("square128", None, 1111, 1300, 200),              # a chunk a tile
    ("square128", None, 2500, 2500, 257),              # two
    ("square128", None, 1300, 2100, 700),              # three; a tile a workgroup
    ("square128", None, 3001, 2999, 1100),             # more tiles than workgroups
    ("square128", None, 4200, 4200, 1025),
    ("square256", None, 4000, 4050, 200),
    ("square256", None, 3900, 4095, 500),
    ("square256", None, 7900, 4090, 700),              # more tiles than workgroups
    ("square256", None, 8100, 8100, 1300),
]
