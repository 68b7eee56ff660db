"""Sizes of 8-bit layers and of projections with adapters, each with the kernel that it is meant for: the GPU tests run them, a host test checks that the
library's choice of a kernel still gives them these, so that a new estimate of the times does not leave a kernel without a test."""

# Projections whose adapters' share goes through memory, by a table of `n` adapters: (M, N, K, n, rank, weights, group), the kernel that adds it.  The rows ask
# for two of them only; with a table of these two the same rows are computed in the tiles, but on packed tiles of 128 x 256 and on unpacked weights.
SHARE = [
    ((115, 1000, 600, 40, 24, "f16", 0), "rows_tile_kernel<0,1,64,32,2,1,3,4>"),
    ((10, 8200, 264, 9, 24, "f16", 0), "rows_tile_kernel<0,1,64,64,2,2,3,2>"),
    ((300, 4104, 1032, 40, 72, "f16", 0), "rows_tile_kernel<0,1,128,64,4,1,3,2>"),
    ((700, 4104, 264, 40, 40, "f16", 0), "rows_tile_kernel<0,1,128,128,2,2,3,1>"),
    ((1500, 4104, 1032, 90, 24, "f16", 0), "rows_tile_kernel<0,1,128,256,2,4,3,1>"),
    ((1100, 10248, 1288, 90, 40, "f16", 0), "moe_pp_kernel<0,0,0,1>"),
    ((10, 12296, 264, 16, 128, "w4", 128), "shared_rows_kernel<1,0,0,1,2,1,4,2,3,1>"),
    ((40, 4104, 520, 40, 72, "w4", 32), "shared_rows_kernel<1,0,0,4,2,1,4,2,3,1>"),
    ((103, 16, 280, 52, 8, "w4", 64), "shared_rows_kernel<1,0,0,2,2,1,2,4,3,1>"),
    ((100, 4104, 264, 40, 24, "w4", 64), "shared_rows_kernel<1,0,0,2,2,1,4,2,3,1>"),
    ((300, 8200, 264, 40, 24, "w4", 32), "shared_rows_kernel<1,0,0,4,4,1,8,1,3,1>"),
    ((300, 8200, 264, 40, 24, "w4", 64), "shared_rows_kernel<1,0,0,2,4,1,8,1,3,1>"),
    ((400, 4104, 264, 40, 24, "w4", 128), "shared_rows_kernel<1,0,0,1,4,1,8,1,3,1>"),
    ((500, 12296, 264, 40, 24, "w4", 32), "shared_rows_kernel<1,0,0,4,8,2,8,1,3,1>"),
    ((500, 12296, 264, 40, 24, "w4", 64), "shared_rows_kernel<1,0,0,2,8,2,8,1,3,1>"),
    ((500, 12296, 264, 40, 24, "w4", 128), "shared_rows_kernel<1,0,0,1,8,2,8,1,3,1>"),
    ((2207, 256, 3696, 9, 88, "w4", 32), "rows_tile_kernel<0,1,64,64,2,2,3,2>"),
    ((4752, 344, 3800, 5, 32, "w4", 128), "rows_tile_kernel<0,1,128,64,4,1,3,2>"),
    ((1950, 1040, 1064, 58, 16, "w4", 64), "rows_tile_kernel<0,1,128,128,2,2,3,1>"),
    ((2901, 4232, 152, 5, 80, "w4", 128), "rows_tile_kernel<0,1,128,256,2,4,3,1>"),
    ((1300, 10248, 1288, 90, 40, "w4", 32), "moe_pp_kernel<0,0,0,1>"),
]

# The same, computed in the tiles.
_FEW_W4 = {32: (4, 2, 2), 64: (2, 3, 2), 128: (1, 3, 2)}  # groups of a step, register sets with one and with two tiles of columns
IN_TILES = [
    ((40, 520, 1032, 3, 24, "f16", 0), "few_rows_kernel<0,0,0,1,1,8,3,1>"),
    ((11, 4672, 520, 5, 40, "f16", 0), "few_rows_kernel<0,0,0,1,2,8,3,1>"),
    ((115, 1000, 600, 2, 72, "f16", 0), "rows_tile_kernel<0,2,64,32,2,1,3,4>"),
    ((10, 8200, 264, 3, 24, "f16", 0), "rows_tile_kernel<0,2,64,64,2,2,3,2>"),
    ((300, 4104, 1032, 3, 72, "f16", 0), "rows_tile_kernel<0,2,128,64,4,1,3,2>"),
    ((700, 4104, 264, 3, 40, "f16", 0), "rows_tile_kernel<0,2,128,128,2,2,3,1>"),
    ((1500, 4104, 1032, 3, 24, "f16", 0), "rows_tile_kernel<0,2,128,256,2,4,3,1>"),
    ((1100, 10248, 1288, 3, 96, "f16", 0), "moe_pp_kernel<0,0,0,2>"),
    ((19742, 1032, 520, 2, 24, "f16", 0), "moe_pp_kernel<0,0,0,2>"),
]
for _group, (_ng, _one, _two) in _FEW_W4.items():
    IN_TILES += [
        ((40, 520, 1032, 3, 24, "w4", _group), "few_rows_kernel<1,0,0,%d,1,8,%d,1>" % (_ng, _one)),
        ((9, 4672, 520, 5, 40, "w4", _group), "few_rows_kernel<1,0,0,%d,2,8,%d,1>" % (_ng, _two)),
        ((66, 24, 440, 2, 8, "w4", _group), "shared_rows_kernel<1,0,0,%d,2,1,2,4,3,1>" % _ng),
        ((40, 4104, 520, 3, 72, "w4", _group), "shared_rows_kernel<1,0,0,%d,2,1,4,2,3,1>" % _ng),
        ((300, 8200, 264, 3, 24, "w4", _group), "shared_rows_kernel<1,0,0,%d,4,1,8,1,3,1>" % _ng),
    ]

# 8-bit layers on 256 x 256 tiles: one round and several, six rows in the last row block, eight columns in the last tile, reductions that end inside a step,
# one of a single step.
Q8_LARGE = [(262, 22344, 1296), (527, 13456, 1296), (19742, 1032, 1040), (4365, 16688, 144), (16866, 8200, 16)]

# Weights on both sides of 2 GiB, (N, K) of E4M3 and of FP16 ones: 256 x 256 tiles address them with 31 bits and give way beyond.
Q8_WEIGHTS, F16_WEIGHTS = ((131064, 16384), (131080, 16384)), ((65528, 16384), (65544, 16384))
