"""Sizes at which the linear layers' calls choose each of their tiles, for tests of what depends on the tile."""

# (tile, tokens, inputs, outputs, the weight by rows of outputs): each tile with both layouts, and with outputs that fill whole lines of 128 bytes (64
# divides them) and not
ON_TILES = [
    (0, 2, 784, 4560, False), (0, 1, 776, 4160, True), (1, 1, 200, 8448, False), (1, 1, 256, 8416, True), (2, 35, 264, 2048, False), (2, 97, 200, 2080, True),
    (3, 33, 96, 1336, False), (3, 33, 96, 2816, True), (4, 2830, 992, 72, False), (4, 161, 896, 2048, True), (5, 67, 472, 8576, False), (5, 65, 472, 8376, True),
    (6, 65, 104, 8456, False), (6, 65, 136, 8896, True), (7, 139, 344, 10936, False), (7, 131, 352, 10944, True), (8, 131, 96, 11648, False), (8, 136, 96, 11352, True),
    (9, 258, 160, 11032, False), (9, 262, 136, 11264, True), (10, 916, 136, 7872, False), (10, 1176, 136, 6280, True), (11, 1289, 96, 5904, False),
    (11, 651, 104, 11008, True), (12, 1357, 96, 8320, False), (12, 1013, 104, 9656, True), (13, 1, 96, 8, False), (13, 17, 96, 64, True), (14, 5, 776, 64, False),
    (14, 3, 264, 8, True)]

# (tokens, inputs, outputs, layout): few tiles and a long sum, whose ranges are joined
IN_RANGES = [(1, 7184, 544, True), (33, 5520, 5584, False), (2, 7168, 120, True), (1062, 4056, 8, False), (1, 5152, 8, True), (17, 8200, 264, False), (129, 7744, 336, True)]

# (tokens, outputs, inputs, the weight, its gradient by rows of outputs): backward passes both of whose products are split, the ranges of dx or of dw the longer part
# of the workspace
BACKWARD_IN_RANGES = [(2202, 2648, 8, True, False), (2050, 2888, 8, True, True), (1995, 2176, 40, True, True), (2643, 1848, 72, True, False), (2569, 3856, 24, False, True),
                      (2114, 2896, 40, False, False), (1857, 3336, 40, False, True)]
