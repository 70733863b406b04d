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

# results in fp32, whose codes are widened: none on 256 x 256 tiles, nor on 128 x 128 ones through registers
WIDENED = [
    ((8100, 4000, 2064, None, True, 0, 0), (128, 1, True)), ((8100, 4001, 2050, "silu", True, 1, 3), (128, 1, True)),
    ((4099, 2040, 4112, "gelu", True, 16, 16), (128, 1, True)), ((8200, 2048, 640, "relu", True, 0, 0), (128, 1, True)),
    ((1000, 2001, 16_400, None, True, 0, 0), (128, 2, True)), ((300, 8192, 20_000, "silu", True, 0, 0), (128, 2, True)),
    ((600, 2040, 40_016, None, True, 0, 0), (128, 6, True)), ((600, 2040, 40_016, "relu", True, 0, 0), (128, 3, True)),
    ((4099, 1000, 1024, None, True, 0, 0), (64, 1, True)), ((600, 600, 8192, "gelu", True, 0, 0), (64, 4, True)),
    ((3001, 512, 1000, "silu", True, 0, 0), (64, 1, False)), ((3000, 1023, 1023, None, True, 1, 1), (64, 1, False)),
    ((8100, 4000, 2064, "silu", True, 16, 1), (64, 1, False)), ((260, 520, 16_400, None, True, 16, 1), (64, 15, False)),
]
# results in bf16 on smaller tiles
SMALLER = [
    ((4099, 4000, 4112, None, False, 0, 0), (128, 1, True)), ((1000, 2001, 16_400, "silu", False, 0, 0), (128, 1, True)),
    ((512, 2048, 65_536, None, False, 0, 0), (128, 4, True)), ((8100, 4000, 2064, "gelu", False, 16, 1), (128, 1, False)),
    ((512, 2048, 65_536, "silu", False, 16, 1), (128, 4, False)), ((3000, 1023, 1023, None, False, 0, 0), (128, 1, False)),
    ((2048, 1024, 2048, None, False, 0, 0), (64, 1, True)), ((260, 520, 16_400, "relu", False, 0, 0), (64, 3, True)),
    ((3001, 512, 1000, None, False, 1, 1), (64, 1, False)), ((260, 520, 16_400, "gelu", False, 16, 1), (64, 6, False)),
]
ALL = HUGE + WIDENED + SMALLER
