"""Sizes that the rules send to each kernel of the dense layer, none of them a whole number of tiles, of slabs or of pieces: test_kernel_choice_host.py
asks the rules, the GPU tests run them."""
TILES = ("256x256", "192x256", "128x192", "128x128", "64x128", "64x64")
FEW = -1
# M, m, n; an epilogue that does more than add the bias?; the tile, and the pieces of the contraction
DENSE_FORWARD = [
    ((12321, 776, 200), False, 0, 1), ((13123, 776, 200), True, 0, 1), ((12575, 392, 200), False, 1, 1), ((13097, 520, 200), True, 1, 1), ((11059, 264, 200), False, 2, 1),
    ((13101, 264, 200), True, 2, 1), ((10921, 136, 1032), False, 3, 1), ((12357, 200, 200), True, 3, 1), ((1379, 2312, 776), True, 3, 1), ((10889, 136, 200), False, 4, 1),
    ((5377, 648, 200), True, 4, 1), ((65, 136, 200), False, 5, 1), ((65, 136, 200), True, 5, 1), ((12605, 776, 2312), True, 0, 1), ((12608, 768, 2296), True, 1, 1),
    ((129, 2088, 2120), False, 5, 2), ((95, 2712, 1864), True, 5, 2), ((463, 216, 1288), False, 5, 3), ((65, 136, 840), True, 5, 3), ((33, 136, 968), True, 5, 4),
    ((17, 136, 1528), False, 5, 6), ((1, 136, 2424), True, 5, 8), ((5, 136, 200), True, FEW, 1), ((17, 136, 200), True, FEW, 1), ((33, 136, 200), True, FEW, 1)]
# M, m, n; the values that make dZ (one without an activation or with relu, three otherwise); everything behind dZ in one launch?; the tile of dW, and whether the rows are cut into pieces
DENSE_BACKWARD = [
    ((3555, 4120, 904), 1, False, 256, True), ((97, 3336, 2312), 1, False, 256, False), ((3215, 136, 2200), 1, False, 128, True), ((97, 4104, 200), 1, False, 128, False),
    ((1185, 136, 200), 1, False, 64, True), ((97, 2504, 200), 1, False, 64, False), ((97, 136, 200), 1, True, 64, False),
    ((8025, 136, 2952), 3, False, 256, True), ((12613, 2312, 776), 3, False, 256, True), ((97, 3592, 2184), 3, False, 256, False), ((935, 4120, 200), 3, False, 128, True),
    ((97, 3592, 520), 3, False, 128, False), ((801, 136, 200), 3, False, 64, True), ((97, 1384, 200), 3, False, 64, False), ((97, 136, 200), 3, True, 64, False)]
# N, pixels, C, groups: with the forward and the backward in both types, every kernel of the group norm
GROUP_NORM = [(1, 1, 8, 1), (1, 1, 8, 2), (1, 1, 8, 4), (1, 1, 520, 1), (1, 17, 136, 1), (1, 17, 136, 2), (1, 17, 136, 4), (1, 17, 264, 1), (1, 33, 136, 2), (1, 33, 136, 4), (1, 33, 264, 1),
              (1, 33, 264, 2), (1, 33, 264, 4), (1, 65, 264, 1), (1, 65, 264, 2), (1, 65, 264, 8), (257, 259, 136, 1), (257, 131, 264, 2), (259, 261, 136, 8), (521, 33, 264, 1)]
