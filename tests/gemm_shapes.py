"""Sizes at which the matrix products' kernels run as they do in large calls: several tiles a pair of CTAs in every
form and width, rings that turn, large float32 tiles. test_gemm_plan.py shows which size reaches what."""

# (M, K, F, N) of a whole gated block: on 16-byte boundaries, and off them
BLOCKS = [(1072, 784, 4896, 832), (4912, 1096, 808, 2088), (1072, 776, 2504, 808), (2768, 1640, 1040, 4024), (1368, 920, 5848, 1448),
          (4976, 456, 960, 2568), (1000, 464, 1920, 4960), (3080, 3824, 656, 1928), (3080, 432, 2848, 1376), (2072, 4280, 608, 816),
          (1072, 424, 3624, 3544), (2624, 432, 4896, 480), (4168, 584, 1032, 3880), (4216, 3064, 880, 2064)]
ODD_BLOCKS = [(4983, 789, 915, 978), (1092, 910, 5517, 821), (3361, 2574, 798, 3189), (1604, 458, 5852, 1813)]
# (M, K, N) of a product with all that its end reads and writes
PROJECTS = [(3000, 640, 2560), (3176, 704, 3088), (2049, 905, 5003), (4267, 849, 2050), (4093, 520, 5120)]
# (M, K, N) of few rows, and of a gated pair
FEW = [(1, 65600, 2000), (17, 8200, 20000), (70, 20000, 9000), (128, 12000, 5000), (33, 1096, 128256)]
FEW_GATED = [(1, 8192, 7000), (64, 20008, 4100), (100, 4096, 14336), (128, 30000, 600), (5, 1500, 19000)]


def products(M, K, F, N):
    """The products of a gated block's forward and backward pass: form, rows, columns, summed index."""
    return [("gated", M, F, K), ("plain", M, N, F), ("grad", M, F, N), ("columns", N, F, M), ("rows", M, K, 2 * F), ("twice", F, K, M)]
