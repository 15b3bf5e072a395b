"""Sizes that reach every variant of the kernels around MXFP4 experts.  The GPU tests run them; a CPU test asks the launches themselves which variant each
one takes, so that a changed rule cannot quietly leave a variant untested."""

# T, k, E, N, K of the matvec: its work-groups are (N / 64, rounded up) * min(T k, E), so many that four row tiles share one, in fp32 and in bf16
MATVEC_FOUR_TILES = [
    (16, 6, 64, 272, 160),           # two slots an expert on average, the last row tiles cut off
    (16, 16, 40, 464, 96),           # more than 16 slots of one expert
    (16, 2, 1, 16400, 64),           # 32 slots of the only expert
    (1, 6, 64, 5520, 64),
    (2, 8, 64, 2064, 128),
    (4, 4, 16, 2096, 320),
    (5, 3, 9, 1872, 1408),           # fp32: slots taken apart for the work-group up to two, lane by lane from three on
    (3, 1, 1, 32784, 96),            # no indices
    (7, 2, 2, 8208, 544),
]
# the same with few work-groups: one row tile and eight waves
MATVEC_ONE_TILE = [(1, 6, 64, 64, 2048), (16, 16, 5, 32, 96), (16, 1, 1, 48, 1408)]

# T, k, E, N, K of the product, by tile shape (32 x 128, 64 x 128, 128 x 256) and by how work-groups find their slots; two lengths of K each, the second a multiple
# of 128 (its rows' scales begin on dwords)
PRODUCT_SEARCH = [
    ((300, 4, 20, 1040, 96), (150, 4, 20, 1040, 128)),
    ((1000, 4, 20, 1040, 352), (1600, 2, 12, 1040, 128)),
    ((3000, 2, 30, 1040, 160), (2000, 4, 12, 1040, 384)),
]
PRODUCT_LIST = [
    ((5000, 2, 8, 48, 96), (100, 6, 64, 2832, 128)),
    ((800, 6, 64, 2832, 96), (800, 6, 64, 2832, 128)),
    ((4600, 2, 40, 2064, 160), (2048, 4, 60, 2832, 128)),
]
PRODUCT_PLAIN = [                    # no indices
    ((300, 1, 1, 272, 96), (300, 1, 1, 272, 256)),
    ((1600, 1, 1, 2064, 96), (1600, 1, 1, 2064, 128)),
    ((4100, 1, 1, 2064, 96), (4100, 1, 1, 2064, 640)),
]

# E, n_group, topk_group, k of routings that sixteen lanes decide (from 2049 tokens on) while the last lane or lanes have no experts
ROUTE_PART_LANES = [(4, 1, 1, 4), (12, 1, 1, 3), (60, 1, 1, 4), (100, 1, 1, 8), (132, 1, 1, 6), (204, 1, 1, 16), (160, 5, 2, 6), (160, 10, 3, 8), (96, 3, 2, 5), (80, 10, 10, 16), (24, 3, 1, 8)]
# and of those whose groups are not a power of two of whole lanes: a wave per token
ROUTE_ODD_GROUPS = [(160, 8, 3, 6), (160, 2, 1, 8), (60, 6, 2, 4), (66, 1, 1, 6)]
ROUTE_TOKENS = 2053
