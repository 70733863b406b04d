"""Products of 8-bit floating point codes by the tiles that they run on: (rows, outputs, depth, gate, fp32 results, pad, shift)
and (side of the tiles, workgroups that share a depth, operands straight to LDS).  pad and shift lay the operands' rows at 16
bytes (0) or not.  Whole tiles and tails in every direction: rows and outputs that end inside a tile, an outputs' row at no
16 bytes, a depth that ends inside a block of scales, one that is copied to aligned rows, one that is split."""

HUGE = [
    ((8100, 4000, 2064, None, False, 0, 0), (256, 1, True)), ((8100, 4000, 2064, "silu", False, 0, 0), (256, 1, True)),
    ((4099, 2040, 4112, None, False, 0, 0), (256, 1, True)), ((8200, 1000, 4112, None, False, 16, 16), (256, 1, True)),
    ((4099, 4000, 4112, "gelu", False, 0, 0), (256, 1, True)), ((8200, 2040, 2064, "relu", False, 16, 16), (256, 1, True)),
    ((8100, 4001, 2050, None, False, 0, 0), (256, 1, True)), ((8100, 4001, 2050, "silu", False, 1, 3), (256, 1, True)),
    ((20_011, 4096, 1024, "silu", False, 0, 0), (256, 1, True)), ((4096, 4096, 4096, None, False, 0, 0), (256, 1, True)),
    ((300, 8192, 20_000, None, False, 0, 0), (256, 4, True)), ((300, 8192, 20_000, "gelu", False, 0, 0), (256, 2, True)),
    ((600, 2040, 40_016, "silu", False, 0, 0), (256, 4, True)),
]
