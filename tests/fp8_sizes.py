"""Sizes that take each kernel of the 8-bit floating-point linear: the launch-plan test asserts that they do, the GPU test runs them."""

# Streaming kernel, (rows, channels) of a tile: [(rows, K, channels)]; one tile of rows and several, one row and one short of whole ones,
# blocks of 128 fewer, as many and more than its eight waves take in turn, the last one partial
STREAM = {
    (16, 16): [(1, 16, 16), (1, 896, 112), (1, 1040, 96), (1, 4240, 48), (47, 2144, 48), (17, 272, 16)],
    (16, 32): [(1, 16, 8304), (1, 1040, 4176), (15, 2144, 4112), (17, 1168, 2096)],
    (16, 64): [(1, 1040, 14544), (15, 2144, 10864)],
    (32, 32): [(33, 896, 3408), (31, 1040, 4720), (33, 4240, 2800)],
    (32, 64): [(31, 16, 8272), (31, 1040, 8400), (31, 4240, 8208)],
    (64, 32): [(65, 16, 3376), (65, 1040, 3344), (65, 2144, 3344)],
    (64, 64): [(65, 16, 5584), (65, 896, 5520), (65, 2144, 5584), (63, 1040, 8400)],
}
# Tiled kernel, (rows, channels, groups of waves): one row more than whole tiles, the last channel tile partly past the last channel; one
# K-step, as many as the ring has stages, one fewer and one more, the last one partial; an odd number of them for two groups
TILED = {
    (64, 128, 1): [(65, 16, 8336), (65, 256, 8208), (65, 384, 8208), (65, 400, 8208)],
    (64, 128, 2): [(65, 3216, 8208), (65, 3792, 8336), (65, 5248, 8208)],
    (128, 128, 1): [(1279, 16, 2448), (129, 384, 15632), (129, 512, 13808), (129, 592, 12432)],
    (256, 128, 1): [(257, 16, 13168), (257, 256, 13072), (257, 400, 13072)],
    (256, 256, 1): [(513, 16, 14608), (513, 128, 14576), (513, 256, 14576), (513, 336, 14576)],
}
# 256 x 256 tiles of which those behind whole rounds are taken in halves: 10 of them, of 16 channels (the second halves hold none) and of
# 144; one; many
HALVES = [(2049, 272, 14608), (2049, 144, 14480), (2049, 400, 14576), (1281, 1168, 11920)]
