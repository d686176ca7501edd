"""The sizes of block_tiles.py reach every tile, without a GPU."""
import os
import subprocess

import block_tiles as tiles

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_tile_is_reached(tmp_path):
    exe = str(tmp_path / "block_tile_choice")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", os.path.join(ROOT, "tests", "native", "block_tile_choice.cpp"), "-o", exe], check=True)
    asked = [(kind, "gated %d %d %d %d %d %d" % (tiles.KINDS[kind], *case)) for kind, cases in tiles.GATED.items() for case in cases]
    asked += [(None, "ortho %d %d %d" % case) for case in tiles.ORTHOGONAL]
    r = subprocess.run([exe], input="\n".join(q for _, q in asked) + "\n", capture_output=True, text=True, timeout=60)
    lines = r.stdout.splitlines()
    assert r.returncode == 0 and len(lines) == len(asked)
    gated, ortho = set(), set()
    for (kind, _), line in zip(asked, lines):
        first, *rest = line.split()
        if kind:
            gated |= {(kind, first.split(":")[1], tile) for tile in rest}
        else:
            ortho |= {first + " " + tile if tile.startswith("update") else tile for tile in rest}
    want_gated, want_ortho = tiles.wanted()
    assert want_gated <= gated, sorted(want_gated - gated)
    assert want_ortho <= ortho, sorted(want_ortho - ortho)
