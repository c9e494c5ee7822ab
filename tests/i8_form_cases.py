"""Shapes that reach each kernel form of the products of 8-bit integers, with a remainder in every dimension.  Shared by the CPU test, which asks for the form, and the GPU
test, which runs them."""


def up(n, to):
    return (n + to - 1) // to * to


# form, M, N, K
FORMS = [("few_rows_16x16", 5, 1000, 300), ("few_rows_16x32", 15, 32 * 300 - 3, 200), ("few_rows_16x32", 16, 9000, 4500), ("few_rows_16x64", 13, 64 * 258 - 35, 200), ("few_rows_16x64", 16, 64 * 256, 9001), ("few_rows_32x16", 29, 1000, 1100), ("few_rows_32x32", 30, 9000, 520),
         ("few_rows_32x64", 77, 16 * 513 + 5, 260), ("128x128", 300, 9000, 390), ("128x128", 1500, 1300, 1170), ("256x256", 4000, 2300, 700), ("256x256", 2500, 6000, 130), ("256x256_long", 4093, 4091, 4099), ("256x256_long", 4096, 5000, 4096)]
# form, rows of each expert, N, K
GROUPED = [("few_rows_16x16", [3, 0, 5, 1], 500, 260), ("few_rows_32x16", [20, 17, 19, 20], 1000, 200), ("few_rows_32x32", [18] * 30, 520, 150), ("128x128", [100, 0, 333, 20, 150], 2500, 400),
           ("256x256", [1000, 300, 2100, 7], 2300, 260), ("256x256_long", [4000, 0, 300, 8100, 7], 2300, 4500)]
