"""The example that runs the sampled mean and both class losses together: it learns, in every type."""
import json
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_step_learns(dtype):
    r = subprocess.run([sys.executable, "-m", "paper_2511_13645_amd.entity_step", "--nodes", "3000", "--dim", "64", "--batch", "256",
                        "--slots", "8", "--steps", "30", "--dtype", dtype], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    line = json.loads(r.stdout.strip().splitlines()[-1])
    assert line["last_loss"] < line["first_loss"]
