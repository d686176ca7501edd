"""How long the plans of the block's products take a launch to be, without a GPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_job_of_a_launch_counts(tmp_path):
    exe = str(tmp_path / "block_span_check")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Xlinker", "--no-as-needed", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    os.path.join(ROOT, "tests", "native", "block_span_check.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr
