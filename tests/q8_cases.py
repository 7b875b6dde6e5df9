"""Sizes of products in 8 bits by the kernel that each is chosen for; tests/test_q8_plan.py holds the estimate to them."""

# Tile kernels, undivided, with more steps of 128 k than twice the stages in LDS: shape -> (rows, k, channels).  Steps are 7 (k = 805:
# rows that are copied to aligned ones first), 9 (1040) and 16 (2000), none with a whole last step.
RING = {0: [(1175, 805, 10058), (1200, 1040, 10058), (3006, 2000, 4100)],     # 256 channels x 256 rows
        1: [(3608, 805, 2050), (3909, 1040, 2050), (805, 2000, 10058)],       # 256 x 192
        2: [(583, 805, 10058), (805, 1040, 7002), (2404, 2000, 2498)],        # 256 x 128
        3: [(657, 805, 7002), (1138, 1040, 4100), (694, 2000, 7002)],         # 128 x 192
        4: [(287, 805, 10058), (546, 1040, 7002), (953, 2000, 4100)],         # 128 x 160
        5: [(324, 805, 4100), (213, 1040, 7002), (620, 2000, 3002)],          # 128 x 128
        6: [(65, 805, 130), (102, 1040, 300), (139, 2000, 130)]}              # 128 x 64
STEPS = {805: 7, 1040: 9, 2000: 16}

# Few-row kernels: channels at which a workgroup takes one, two or four blocks of 16; rows that take one, two or four blocks of 16; widths of
# 18 and 32 steps, which a workgroup's wavefronts take in two to eight trips, the last one of 2181 not all of them.
FEW_CHANNELS = [520, 8200, 12290]
FEW_ROWS = [1, 16, 17, 32, 33, 64]
FEW_WIDTHS = [2181, 4096]
