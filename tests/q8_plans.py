"""Shapes of the 8-bit product that reach every tile width of the tensor-core form,
each with tiles in one piece, all tiles cut along K, and whole tiles with the
rest cut, from either side; every K passes the operand ring and a fold of the
accumulators. The host test holds them to that, the GPU test to the results."""

# tokens, channels, K, width, form of the work, sides exchanged
PLANS = [
    (9, 19, 6209, 32, "cut", False), (21, 17, 4220, 32, "cut", True),
    (9, 15036, 2640, 32, "one piece", False), (9739, 17, 1429, 32, "one piece", True),
    (9, 19546, 8073, 32, "whole and cut", False), (19812, 19, 2231, 32, "whole and cut", True),
    (34, 34, 14766, 64, "cut", False), (37, 34, 14920, 64, "cut", True),
    (33, 9834, 2105, 64, "one piece", False), (9731, 33, 2313, 64, "one piece", True),
    (33, 19866, 2179, 64, "whole and cut", False), (19538, 34, 3285, 64, "whole and cut", True),
    (68, 258, 14199, 96, "cut", False), (278, 72, 13913, 96, "cut", True),
    (65, 9918, 1268, 96, "one piece", False), (10176, 67, 1383, 96, "one piece", True),
    (65, 19660, 1691, 96, "whole and cut", False), (19591, 71, 3229, 96, "whole and cut", True),
    (225, 302, 10921, 128, "cut", False), (553, 100, 15890, 128, "cut", True),
    (103, 9877, 1273, 128, "one piece", False), (10352, 108, 1279, 128, "one piece", True),
    (208, 11163, 2273, 128, "whole and cut", False), (10475, 202, 2523, 128, "whole and cut", True),
    (144, 583, 11661, 160, "cut", False), (547, 131, 12135, 160, "cut", True),
    (5196, 259, 1264, 160, "one piece", False), (10439, 131, 2462, 160, "one piece", True),
    (442, 6449, 2368, 160, "whole and cut", False), (19728, 132, 1951, 160, "whole and cut", True),
    (166, 1030, 14896, 192, "cut", False), (1167, 166, 15214, 192, "cut", True),
    (179, 9748, 1479, 192, "one piece", False), (9743, 164, 1973, 192, "one piece", True),
    (172, 19626, 2884, 192, "whole and cut", False), (9918, 335, 3453, 192, "whole and cut", True),
    # several whole tiles a pair
    (8192, 800, 784, 160, "one piece", False), (14094, 502, 1887, 192, "one piece", False),
    (4096, 4096, 4096, 160, "whole and cut", False), (3247, 4016, 8645, 192, "whole and cut", False),
]


def row_stride(K):
    """Rows of codes at multiples of 16 bytes."""
    return (K + 15) // 16 * 16
