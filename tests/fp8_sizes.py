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
# Rows quantised in the launch of the linear, (channels of a work-group, rows there is room for): blocks of 128 fewer, as many and more than
# the eight waves take in turn, the last one partial, the last work-group's channels partly past the last one
ROWS16 = {
    (16, 1): [(1, 16, 16), (1, 1040, 4096), (1, 4240, 8208), (1, 2064, 14352)],
    (16, 2): [(2, 1040, 48), (2, 5136, 8208)],
    (16, 4): [(3, 4240, 144), (4, 2048, 14352)],
    (16, 8): [(5, 1040, 112), (8, 2064, 10240)],
    (32, 1): [(1, 16, 4112), (1, 2144, 4112), (1, 4240, 8176)],
    (32, 2): [(2, 1040, 4112)],
    (32, 4): [(3, 400, 8176), (4, 5136, 4144)],
    (32, 8): [(7, 1040, 4112), (8, 5136, 4112)],
    (64, 1): [(1, 16, 8208), (1, 1040, 8240), (1, 2032, 14352)],
    (64, 2): [(2, 1040, 8208)],
    (64, 4): [(3, 400, 8240), (4, 2032, 8208)],
    (64, 8): [(5, 1040, 8208), (8, 4240, 10256)],
}
