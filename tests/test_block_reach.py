"""How far the steps of an orthogonalised update may take singular values, and which steps are taken, without a GPU."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000   # non-null, 16-byte aligned; never dereferenced on an error path
ARG, WORKSPACE = -2, -7


def test_reach_and_units(tmp_path):
    exe = str(tmp_path / "block_reach_check")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Xlinker", "--no-as-needed", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    os.path.join(ROOT, "tests", "native", "block_reach_check.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


@pytest.mark.parametrize("triples,status", [
    ([(8.0, -22.0, 16.5)], WORKSPACE),                       # past the check of coefficients, to the next
    ([(8.0, -23.0, 16.5), (1.766, -0.644, 0.072), (3.4445, -4.775, 2.0315)], WORKSPACE),
    ([(16.0, 16.0, 16.0)], WORKSPACE),
    ([(8.0, 22.0, 16.5)], ARG), ([(0.0, 17.0, 0.0)], ARG), ([(2.0, 0.0, 0.0)] * 3 + [(17.0, 0.0, 0.0)], ARG), ([(0.0, 1025.0, -1025.0)], ARG)])
def test_coefficients(triples, status):
    from paper_2511_13645_amd import binding, build
    if build.is_stale():
        build.build_hip()
    host = (ctypes.c_float * 96)(*(x for t in triples for x in t))
    assert binding.lib().fsa_orthogonalize(FAKE, 0, 32, 0, 1, 64, 32, host, len(triples), 0.0, 1.0, FAKE, None, 1 << 40, None) == status
