"""The sizes of class_tiles.py do what they are there for, by the plan: several tiles a workgroup in every form of the kernels."""
import os
import subprocess

from class_tiles import BOTH, FEW_CLASSES, FEW_ROWS, WIDE

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_sizes_turn_the_loops(tmp_path):
    exe = str(tmp_path / "class_tiles")
    subprocess.run(["g++", "-O1", "-std=c++17", os.path.join(ROOT, "tests", "native", "class_tiles.cpp"), "-o", exe], check=True)
    asked = [(t, v, d, kind, k) for t, v, d in BOTH + FEW_ROWS + FEW_CLASSES + WIDE for kind in (0, 1, 2) for k in (1, 5)]
    lines = "\n".join("%d %d %d %d %d" % (t, v, d, kind + 4 * (kind > 0 and d in (64, 128, 256, 384, 640, 1024)), k) for t, v, d, kind, k in asked)
    out = subprocess.run([exe], input=lines, capture_output=True, text=True, check=True).stdout.split("\n")
    packed = set()
    for (t, v, d, kind, k), line in zip(asked, out):
        fwd_wy, fwd_tiles, bwd_wy, bwd_tiles, laid_out = map(int, line.split())
        what = (t, v, d, kind, k, line)
        if (t, v, d) in BOTH:
            assert fwd_wy == 1 and fwd_tiles >= 3 and bwd_wy == 1 and bwd_tiles >= 3, what
            packed.add((kind > 0, bool(laid_out)))
        elif (t, v, d) in FEW_ROWS:
            assert fwd_tiles >= 3 and fwd_wy == (2 if t == 70 or (kind == 0 and d > 128) else 4), what
        elif (t, v, d) in FEW_CLASSES:
            assert bwd_tiles >= 3 and bwd_wy == (2 if v == 60 or (kind == 0 and d > 128) else 4), what
        else:
            assert fwd_tiles >= 3 and bwd_tiles >= 3, what
    assert packed == {(False, True), (True, True), (True, False)}
