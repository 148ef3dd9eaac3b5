"""Shapes of the 4-bit product that reach every tile width of the block form, with K in one piece and shared among 2, 4
and 8 blocks, from either side, and the form of SM pairs. The host test holds them to that, the GPU test to the
results."""

# tokens, channels, K, width (0: pairs), blocks that share K, sides exchanged
PLANS = [
    (1, 40, 300, 16, 1, False), (16, 20000, 700, 16, 1, False), (13, 9000, 4000, 16, 2, False),
    (9, 3000, 4100, 16, 4, False), (4, 500, 9000, 16, 8, False), (3000, 9, 700, 16, 1, True), (700, 16, 9000, 16, 8, True),
    (17, 129, 65, 32, 1, False), (31, 2500, 5000, 32, 4, False), (30, 600, 3000, 32, 8, False), (2000, 32, 90, 32, 1, True),
    (33, 1023, 800, 64, 1, False), (64, 2000, 8000, 64, 8, False), (50, 4500, 6000, 64, 4, False), (60, 9000, 6000, 64, 2, False),
    (900, 40, 200, 64, 1, True),
    (65, 65, 65, 128, 1, False), (300, 130, 9000, 128, 8, False), (400, 1000, 8000, 128, 4, False),
    (1000, 1000, 9000, 128, 2, False), (129, 3000, 1100, 128, 1, False), (5325, 123, 285, 128, 1, False),
    (1500, 2100, 290, 0, 1, False), (2100, 2400, 33, 0, 1, False), (300, 9000, 1500, 0, 1, False), (12500, 200, 700, 0, 1, False),
]
