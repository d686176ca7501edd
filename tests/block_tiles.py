"""Sizes of the gated block and of orthogonalised matrices that the plans send to every tile that they choose from, in every form: more rows
and columns than one tile's, and neither a multiple of it.  test_block_tiles.py checks on the CPU that they still do (rates that are tuned again
move them), test_gpu_block_tiles.py runs them."""

# (fine, T, D, H, O) by type; between products lie one number of a 16-bit type, or two (small calls, and fine ones)
GATED = {
    "f32": [(False, 67, 73, 69, 73), (False, 8679, 69, 221, 135), (False, 3205, 35, 1221, 71), (False, 699, 133, 845, 467),
            (False, 659, 109, 33, 2719), (False, 1379, 33, 1985, 137)],
    "bf16": [(False, 67, 65, 65, 65), (True, 203, 137, 4413, 133), (False, 1271, 185, 431, 847), (False, 389, 147, 4015, 133),
             (False, 6219, 37, 705, 79), (True, 1011, 37, 4435, 129), (False, 263, 271, 2053, 2355), (True, 7767, 423, 263, 445),
             (False, 2437, 55, 33, 1555), (False, 8765, 33, 85, 829), (True, 581, 55, 4105, 1631), (False, 1239, 115, 5317, 1603)],
    "f16": [(False, 77, 67, 65, 71), (False, 135, 163, 5689, 135), (False, 451, 699, 855, 331), (False, 909, 129, 1751, 161),
            (False, 2975, 35, 1371, 69), (False, 911, 35, 4335, 101), (False, 477, 39, 33, 2067), (False, 2487, 35, 33, 1539),
            (False, 6361, 689, 279, 645), (False, 2463, 107, 135, 1791), (True, 279, 267, 4709, 263), (True, 595, 55, 3967, 1611),
            (False, 1697, 35, 5413, 1191)],
}
# 16-bit operands of a multiple of 8 elements, which products read where they are
IN_PLACE = [(False, 264, 272, 2056, 2352), (False, 1240, 112, 5320, 1608), (True, 1008, 40, 4432, 136), (False, 6216, 40, 704, 80)]

# (matrices, rows, columns)
ORTHOGONAL = [(1, 65, 65), (29, 131, 129), (57, 259, 257), (1, 547, 65), (18, 193, 1291), (57, 261, 267), (42, 1161, 387), (8, 387, 1161),
              (1, 4096, 1024), (8, 960, 4096), (1, 4096, 4096)]

KINDS = {"f32": 0, "bf16": 1, "f16": 2}
TILES = {
    "f32": {"hidden": ["64x64", "128x64", "256x64"], "slopes": ["64x64", "128x64", "256x64"], "product": ["64x64", "128x64", "256x128"]},
    "16": {"hidden": ["64x64", "128x64", "256x128"], "slopes": ["64x64", "128x64", "128x128"], "product": ["64x64", "128x128", "256x256"]},
}


def wanted():
    """Every form of every tile."""
    gated = set()
    for kind in KINDS:
        tiles = TILES["f32" if kind == "f32" else "16"]
        for planes in ("3",) if kind == "f32" else ("1", "2"):
            for name in ("hidden", "slopes"):
                gated |= {(kind, planes, "%s:%s" % (name, t)) for t in tiles[name]}
            for name in ("answer", "shares", "kept", "grads"):
                gated |= {(kind, planes, "%s:%s" % (name, t)) for t in tiles["product"]}
    squares = TILES["16"]["product"]
    ortho = {"%s:%s" % (name, t) for name in ("gram", "parts", "poly") for t in squares}
    ortho |= {"%s update:%s" % (way, t) for way in ("wide", "tall") for t in squares}
    return gated, ortho
