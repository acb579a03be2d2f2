"""Sizes of the 8-bit calls that reach each of their kernels, shared by the GPU tests
that run them and the host test that asks the library which kernels they are."""

# Products (M, N, K); N a multiple of 32, so that every epilogue takes them.  By tile
# (rows x channels): sizes that divide none, K of whole pairs of K tiles; with more
# tiles than a launch has blocks, then with fewer.
WHOLE = [(33, 32, 768), (11855, 1312, 768), (66, 16448, 768), (563, 22208, 768), (258, 16704, 768), (13207, 1056, 768),
         (131, 16960, 768), (773, 18784, 768), (257, 22528, 768), (798, 24640, 768), (275, 24704, 768)]
# the same with one and with two pairs of K tiles
SHORT_K = [(65, 16832, 256), (33, 32832, 256), (129, 16576, 256), (131, 32864, 256), (257, 25152, 256),
           (65, 16544, 512), (33, 33376, 512), (133, 16416, 512), (130, 33472, 512), (257, 24608, 512)]
# rows padded to whole pairs of K tiles: K ends inside a K tile, with more tiles than
# blocks and with fewer
PADDED = [(4466, 3648, 800), (68, 16928, 832), (524, 22688, 832), (258, 16928, 848), (16426, 800, 880), (133, 23776, 800),
          (658, 23776, 800), (273, 22144, 832), (834, 25248, 816), (329, 25440, 784)]
# K ends behind the first of a pair of K tiles
PADDED_HALF = [(4698, 3392, 896), (69, 17088, 896), (517, 22048, 896), (13370, 1056, 896), (131, 22432, 896),
               (776, 19104, 896), (274, 22432, 896), (778, 25184, 896), (258, 24896, 896)]
# less than a K tile, one, and a little more
PADDED_SHORT = [(9244, 800, 48), (777, 9312, 128), (781, 9248, 144), (257, 19744, 48), (260, 19744, 128), (66, 32800, 144),
                (193, 24672, 48), (196, 24608, 128), (129, 21984, 144), (130, 32992, 48), (130, 33088, 128),
                (129, 33280, 144), (258, 26336, 48), (261, 26656, 128), (268, 24608, 144)]
SPLIT = [(33, 32, 912), (70, 2272, 4096), (5, 9184, 7168), (4111, 32, 10240), (4271, 160, 10240), (134, 12512, 11264)]
# weights straight into registers: 16 or 32 rows, 8 or 4 wavefronts a strip
FEW = [(1, 1536, 1024), (3, 6176, 4096), (16, 4128, 2064), (17, 4096, 2048), (32, 6400, 1296), (9, 6208, 4000)]
# decoder projections between the measured batch sizes
DECODERS = [(1919, 4128, 2064), (638, 24576, 4096), (512, 4096, 12288), (1023, 4096, 12288), (1275, 4096, 12288),
            (4, 5120, 2048), (10, 4096, 4096)]
PRODUCTS = WHOLE + SHORT_K + PADDED + PADDED_HALF + PADDED_SHORT + SPLIT + FEW + DECODERS

# Expert layers: rows, experts, experts of a row, d_model, expert_ffn, and how many of
# the pairs go to expert 1 (so that it has whole row tiles) beside their even share.
EXPERTS = [(1, 128, 8, 2048, 768, 0), (12, 16, 4, 1040, 528, 0),
           # 128 x 128 tiles, whole and short last K tiles
           (40, 16, 4, 1024, 512, 0), (600, 16, 2, 1024, 512, 400), (600, 16, 2, 1040, 528, 400), (400, 8, 1, 1040, 256, 0),
           (400, 8, 1, 256, 144, 300),
           # 128 x 256 in both products, in gate/up or in down alone
           (400, 128, 8, 2048, 768, 0), (976, 128, 8, 2048, 768, 0), (400, 128, 8, 1040, 528, 300), (300, 64, 6, 1024, 1408, 0),
           (500, 60, 4, 1296, 1280, 290), (700, 64, 8, 1456, 768, 400), (400, 128, 8, 1040, 256, 0), (400, 128, 8, 2048, 144, 300),
           # 256-row tiles: some 700 and 1800 rows an expert, K that ends on a K tile and inside one
           (1500, 4, 2, 256, 128, 0), (1500, 4, 2, 272, 144, 0), (3000, 5, 3, 1040, 528, 0), (3000, 5, 3, 1024, 720, 0),
           (2000, 128, 8, 2048, 768, 0), (2100, 16, 8, 528, 272, 0),
           # lists in launches of their own, beside 128-row tiles, too
           (6000, 12, 3, 272, 144, 0), (2600, 256, 8, 256, 128, 300), (2600, 256, 8, 1296, 272, 300)]
