"""Shapes that reach each kernel form of the products of 8-bit integers, with a remainder in every dimension.  Shared by the CPU test, which asks for the form, and the GPU
test, which runs them."""


def up(n, to):
    return (n + to - 1) // to * to


# form, M, N, K: sums of one k step of 128 and less, of as many as the wavefronts' stages hold, and of more
FORMS = [("few_rows_16x16", 5, 1000, 300), ("few_rows_16x16", 16, 700, 9001), ("few_rows_16x16", 29, 900, 9088), ("few_rows_16x16", 3, 301, 100), ("few_rows_16x64", 13, 64 * 258 - 35, 200),
         ("few_rows_16x64", 15, 9000, 4500), ("few_rows_16x64", 16, 64 * 256, 9001), ("few_rows_32x16", 61, 2000, 3333), ("few_rows_32x16", 70, 900, 1300), ("few_rows_32x32", 30, 9000, 520),
         ("few_rows_32x64", 77, 4000, 5000), ("few_rows_32x64", 90, 3900, 1000), ("few_rows_64x64", 130, 4100, 900), ("few_rows_64x64", 200, 3000, 5001), ("few_rows_128x64", 1500, 700, 1031), ("few_rows_128x64", 390, 4001, 9000), ("few_rows_128x64", 1500, 1300, 1170), ("few_rows_128x64", 900, 1900, 1300),
         ("128x128", 300, 9000, 390), ("128x128", 2500, 3000, 1170), ("256x256", 4000, 6000, 700), ("256x256", 2500, 6000, 130), ("256x256_long", 4093, 4091, 4099), ("256x256_long", 4096, 5000, 4096)]
# form, rows of each expert, N, K
GROUPED = [("few_rows_16x16", [3, 0, 5, 1], 500, 9000), ("few_rows_16x64", [3, 0, 5, 1], 500, 260), ("few_rows_16x64", [18] * 30, 520, 150), ("few_rows_32x32", [20, 17, 19, 20], 1000, 2200),
           ("few_rows_32x32", [1, 119], 1000, 3000), ("few_rows_64x64", [299, 0, 1], 2000, 1300), ("few_rows_32x64", [259, 1], 1500, 2100), ("few_rows_64x64", [500, 0, 100, 99, 1], 1400, 1200), ("few_rows_128x64", [100, 399, 1], 2500, 5003), ("128x128", [100, 0, 333, 20, 150], 2500, 400),
           ("256x256", [3000, 300, 6100, 7], 4300, 260), ("256x256_long", [4000, 0, 300, 8100, 7], 2300, 4500)]
