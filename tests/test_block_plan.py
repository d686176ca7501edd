"""The plans of the norm, the gated block and the orthogonalised update without a GPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_workspaces_hold_what_the_plans_put_there(tmp_path):
    exe = str(tmp_path / "block_plan_check")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Xlinker", "--no-as-needed", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    os.path.join(ROOT, "tests", "native", "block_plan_check.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr
