"""Cases of the grouped products and the kernel each is meant to reach, shared by
the GPU tests that run them and the CPU test that looks which kernel a call takes.

A group's size is given in rows; what the library goes by is their mean, rounded
up. KERNELS names the kernels by what stands in their symbols."""
KERNELS = {
    "few16": "k_group_product_few.*Li1ELi4E", "few64": "k_group_product_few.*Li4ELi4E", "any": "k_group_product_any",
    "t32": "k_group_product_fast.*Li32ELi128E", "t64": "k_group_product_fast.*Li64ELi128E",
    "t256": "k_group_product_fast.*Li256ELi256E",
    "fp8_few16": "k_group_product_fp8_few.*Li1ELi4E", "fp8_few64": "k_group_product_fp8_few.*Li4ELi4E",
    "fp8_any": "k_group_product_fp8_any", "fp8_t32": "k_group_product_fp8_fast.*Li32ELi128E",
    "fp8_t64": "k_group_product_fp8_fast.*Li64ELi128E", "fp8_t256": "k_group_product_fp8_fast.*Li256ELi256E",
    "outer_any": "k_group_outer_any", "outer128": "k_group_outer_fast.*Li128ELi128E", "outer256": "k_group_outer_fast.*Li256ELi256E",
}


def spread(mean, groups=16):
    """Sizes around a mean, which they have exactly: an empty group, one of twice the mean, neighbours of tile edges."""
    sizes = [mean] * groups
    for a, b, d in ((0, 1, mean), (2, 3, mean // 2), (4, 5, 1), (6, 7, mean - 1), (8, 9, min(mean, 7))):
        sizes[a] -= d
        sizes[b] += d
    return sizes


# few rows a group with one group of several row tiles, 70 groups
UNEVEN = [50] + [0, 1, 2, 3] * 17 + [5]

# kernel, sizes, n, k, transposed. The kernels of few rows take 16 blocks of K a
# pass, of 64 elements (8 bits: of 128): K on both sides of one, two and more.
PRODUCTS = [
    ("few16", [1, 2, 0, 16], 72, 2048, False), ("few16", [1, 2, 0, 16], 40, 4096, False), ("few16", [3, 0, 9], 33, 1023, False),
    ("few16", [3, 0, 9], 33, 1025, False), ("few16", [7], 65, 2047, False), ("few16", [16, 16], 24, 3333, False),
    ("few64", UNEVEN, 264, 2048, False), ("few64", UNEVEN, 248, 1288, False), ("few64", UNEVEN, 520, 1032, False),
    ("few64", spread(16), 2048, 2560, False), ("few64", [0] * 15 + [256], 1024, 1280, False),
    ("any", spread(16), 2048, 201, False), ("any", spread(40), 135, 2049, False), ("any", spread(40), 1001, 264, True),
    # both sides of the limits of the tiles' heights
    ("t32", spread(17), 2048, 136, False), ("t32", spread(64), 328, 264, False), ("t64", spread(65), 328, 264, False),
    ("t64", spread(127), 2048, 136, False), ("t256", spread(128), 2048, 136, False), ("t256", spread(129), 2048, 72, False),
    ("t64", spread(128), 1792, 136, False),
    ("t32", spread(1), 264, 72, True), ("t32", spread(32), 328, 264, True), ("t64", spread(33), 328, 264, True),
    ("t64", spread(127), 2048, 136, True), ("t256", spread(128), 2048, 136, True), ("t256", spread(300, 10), 2048, 2048, True),
    ("t256", spread(300, 10), 2048, 2048, False),
]

# kernel, sizes, n, k
FP8_PRODUCTS = [
    ("fp8_few16", [1, 2, 0, 8], 72, 4096), ("fp8_few16", [1, 2, 0, 8], 40, 2047), ("fp8_few16", [3, 0, 9], 33, 2049),
    ("fp8_few16", [7], 130, 4333), ("fp8_few16", [8, 8], 24, 6400),
    ("fp8_few64", UNEVEN, 264, 4096), ("fp8_few64", UNEVEN, 264, 2064), ("fp8_few64", UNEVEN, 520, 2176),
    ("fp8_few64", spread(8), 2048, 2320), ("fp8_few64", [0] * 15 + [128], 1024, 4096),
    ("fp8_any", spread(8), 2047, 201), ("fp8_any", spread(40), 135, 2049),
    ("fp8_t32", spread(9), 2048, 144), ("fp8_t32", spread(32), 328, 528), ("fp8_t64", spread(33), 328, 528),
    ("fp8_t64", spread(127), 2048, 144), ("fp8_t256", spread(128), 2048, 144), ("fp8_t256", spread(300, 10), 2048, 2048),
]

# kernel, by their sizes or not, sizes, n, k. Groups of 256 rows and more on the
# average are taken by their size, 64 at a time.
LONG = [0, 1, 2200, 255, 256, 257, 600] + [250 + 3 * (i % 9) for i in range(63)]
OUTERS = [
    ("outer256", True, LONG, 1024, 776), ("outer256", False, spread(255, 32), 1024, 1024), ("outer256", True, spread(256, 32), 1024, 1024),
    ("outer256", True, [300], 4096, 3584), ("outer256", False, [70], 4096, 4096), ("outer256", False, [0], 4096, 4096),
    ("outer128", True, [300], 4096, 2816), ("outer128", False, spread(255, 31), 1024, 1024), ("outer128", True, LONG, 520, 264),
    ("outer256", False, spread(40, 32), 1100 - 4, 1024),
    ("outer_any", True, LONG, 77, 130), ("outer_any", True, [700], 129, 257), ("outer_any", False, spread(40), 1001, 264),
]
