"""Cases of the products of 8-bit integers and the kernel each is meant to reach, shared by the GPU test that runs
them and the CPU test that looks which kernel a call takes: every kernel's loops, and both sides of the limits of a
group's mean size."""
from tests.experts_cases import UNEVEN, spread

KERNELS = {
    "few16": "k_group_product_int8_few.*Li1ELi4E", "few64": "k_group_product_int8_few.*Li4ELi4E", "any": "k_group_product_int8_any",
    "t32": "k_group_product_int8_fast.*Li32ELi128E", "t64": "k_group_product_int8_fast.*Li64ELi128E",
    "t256": "k_group_product_int8_fast.*Li256ELi256E",
}

# kernel, sizes, n, k
PRODUCTS = [
    ("few16", [1, 2, 0, 8], 72, 4096), ("few16", [1, 2, 0, 8], 40, 2047), ("few16", [3, 0, 9], 33, 2049), ("few16", [7], 130, 4333),
    ("few16", [16, 16], 24, 6400), ("few64", UNEVEN, 264, 4096), ("few64", UNEVEN, 264, 2064), ("few64", UNEVEN, 520, 2176),
    ("few64", spread(16), 2048, 2320), ("few64", [0] * 15 + [256], 1024, 4096),
    ("any", spread(8), 2047, 201), ("any", spread(40), 135, 2049), ("any", spread(200, 10), 777, 1001), ("any", spread(17), 264, 392),
    ("t32", spread(17), 2048, 144), ("t32", spread(47), 2048, 144), ("t32", spread(64), 328, 528), ("t64", spread(65), 328, 528),
    ("t64", spread(100, 10), 328, 1040),
    ("t256", spread(48), 2048, 144), ("t256", spread(128), 2048, 272), ("t256", spread(300, 10), 2048, 2048),
]
