"""Sizes that reach every way in which the 4-bit calls are dispatched, each named with that way (test infrastructure): tests/test_mx4_host.py holds
the names to the library's rules, tests/test_gpu_mx4_dispatch.py runs them."""

# m, n, k: an m by n result of sums over k terms.  Tiles of 64 and more take 256 terms a step, and scales for 1024 terms at a time: sums of one
# to four steps, of more, and of some that end within the 1024; ends of rows and columns within a tile.
PRODUCTS = [
    ("16, 4 wavefronts", 100, 77, 513), ("16, 8 wavefronts", 40, 500, 1300), ("16, 16 wavefronts", 33, 64, 7600),
    ("64", 512, 640, 96), ("64", 257, 385, 1281), ("64", 300, 1200, 5000), ("64", 33, 35001, 700),
    ("128", 2001, 1503, 300), ("128", 1001, 2304, 2600), ("128", 700, 5000, 1025),
    ("256", 3000, 4097, 1300), ("256", 3500, 3500, 2300), ("256", 12500, 1000, 200),
]

# m, n, k of a linear layer's gradients, dx [m, k] over n terms and dw [n, k] over m: both by the same tiles, in one launch, or not.
GRADIENTS = [
    ("64", 300, 500, 640), ("64", 511, 450, 1290), ("128", 1001, 1100, 2304), ("256", 3500, 3600, 3501), ("64, 128", 515, 900, 3000),
]

# m, n, k of a linear layer over few rows in one launch: wavefronts and tiles of a workgroup; whether there are further rounds of weights for
# a wavefront, and of values of x for a lane; workgroups for a compute unit.
FEW = [
    ("4 x 1", 1, 300, 1000), ("8 x 1", 9, 333, 1001), ("8 x 1", 3, 300, 4000), ("16 x 1", 1, 300, 5000), ("16 x 1, w, x", 6, 333, 8501),
    ("16 x 1, x", 16, 333, 6101), ("4 x 2", 1, 4100, 1000), ("8 x 2", 8, 4100, 1003), ("8 x 2", 1, 4100, 4096), ("16 x 2", 4, 4100, 4096),
    ("16 x 2, w, x", 5, 4101, 8401), ("8 x 2, x, 2 each", 8, 14336, 4096), ("8 x 2, w, x, 2 each", 4, 8193, 5000), ("4 x 1", 3, 20, 7),
]

# rows, cols of a quantisation along columns: rows of a tile, and whether there is more than one band of 1024 rows.
QUANTISED = [
    ("32", 1001, 768), ("32, bands", 2500, 1000), ("32, bands", 1025, 777), ("64, bands", 5000, 6801), ("64, bands", 5001, 6800),
    ("64", 1000, 33600),
]
