"""Sizes of products in MX4 by the kernel that each is chosen for; tests/test_mx4_launches.py holds the library's choice to them."""

TILE_ROWS = {"128 rows": 128, "64 rows": 64}

# Products grouped by expert on the tile kernels: rows of a tile -> (experts, entries, k, packed channels).  K of one step and of several, with whole
# and partial last blocks, words of scales and steps; 6200 and 6400 are 25 steps, whose scales are dealt out twice.
GROUPED = {"128 rows": [(5, 8000, 300, 300), (40, 5000, 160, 1030), (64, 3000, 520, 600), (3, 4000, 1037, 1030)],
           "64 rows": [(8, 700, 300, 1030), (16, 300, 520, 1030), (64, 700, 1037, 300), (40, 700, 160, 600), (7, 2600, 128, 1400)]}
GROUPED_LONG = {"128 rows": (5, 8000, 6200, 300), "64 rows": (2, 300, 6400, 3002)}

# One matrix on the tile kernels, K of 25 and 27 steps: (rows, k, packed channels)
LONG = {"128 rows": (2500, 6700, 2700), "64 rows": (600, 6200, 3002)}

# Rows at the largest stride, grouped and not; as many as a call by index may have.
FAR = {"rows": (300, 320, 3400), "entries": (2, 300, 320, 3400), "index": (2, 600, 255, 320, 3400)}

# 4.6 GB of weights: (experts, entries, k, channels)
HEAVY = (1024, 12000, 2112, 4096)

# The layers: (experts, choices, tokens, width, hidden) and (rows, width, hidden); both products of each on the tile kernels.
EXPERTS_LAYERS = [(8, 4, 1400, 640, 512), (40, 3, 500, 416, 1000)]
FEEDFORWARD = [(2500, 512, 832), (1100, 1312, 1000)]
