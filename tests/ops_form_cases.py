"""Products with remainders in every dimension, each under the kernel form that it is to run on, on a chip of 256 compute units: E4M3 (rows of each expert, or their number where
nothing is grouped; N, K, type of the result), and the 16-bit forward product and gradients (rows of each expert, N, K).  Sums are long enough for every form's loop to copy ahead of its
multiplications, two k steps and more behind the first."""
import random

EXTRA = 5            # rows without an expert, behind the others


def dealt(T, E, seed=0):
    """T rows dealt to E experts, most of them no multiple of anything."""
    rng = random.Random(seed)
    counts = [0] * E
    for _ in range(T):
        counts[rng.randrange(E)] += 1
    return counts


E4M3 = [
    ("few_rows_16x16", 13, 2039, 1700, "f16"),
    ("few_rows_16x32", 15, 8201, 1300, "f32"),
    ("few_rows_32x16", 30, 2041, 1300, "bf16"),
    ("few_rows_32x32", 29, 8199, 1300, "f32"),
    ("few_rows_32x64", 61, 16391, 1300, "bf16"),
    ("few_rows_16x32", [3, 0, 1, 17, 9] * 3, 4099, 1100, "bf16"),
    ("widened_128x128", 1290, 1310, 1500, "f32"),
    ("widened_128x128", [200, 0, 311, 90], 2501, 1500, "bf16"),
    ("widened_128x128_short_groups", [40, 0, 17, 33, 64, 1] * 4, 4099, 1300, "f32"),
    ("widened_128x128_short_groups", [0] * 12 + [400], 4099, 1300, "f32"),
    ("widened_128x128_two", 3001, 2999, 1300, "f32"),
    ("widened_128x128_two", [70, 90, 0, 131, 128] * 8, 4099, 1300, "f32"),
    ("widened_256x128", 4000, 3990, 2100, "f32"),
    ("widened_256x128", 2047, 3001, 1000, "f32"),
    ("widened_256x128", [1000, 257, 0, 1190, 1001], 4090, 2100, "f32"),
    ("e4m3_128x128", 4730, 4399, 1300, "bf16"),
    ("e4m3_128x128", [70, 90, 0, 131, 128] * 8, 4099, 1300, "f16"),
    ("e4m3_256x256", 8100, 3999, 1300, "bf16"),
    ("e4m3_256x256", [1000, 257, 0, 1500, 1001], 6001, 1300, "f16"),
]
MANY, FEW = dealt(9000, 32), [600, 257, 0, 1, 311]
FORWARD = [
    ("256x256", [2000, 1111, 0, 900], 3999, 1000),
    ("128x256", dealt(4000, 40), 2040, 1000),
    ("128x128", FEW, 1999, 1000),
]
GRAD_A = [
    ("256x256", [2000, 1111, 0, 900], 1000, 3992),
    ("128x128", dealt(4000, 40), 1000, 2040),
]
GRAD_B = [
    ("256x256", MANY, 2040, 1000),
    ("256x256", [1400, 2000, 1111], 3999, 2047),
    ("128x128", FEW, 1999, 1000),
]
# any alignment: rows that are no multiples of 8 elements
UNALIGNED = [("any_alignment_128x128", FEW, 1001, 999), ("any_alignment_128x128", MANY, 2041, 1003)]
