"""The example that runs the sampled mean and both class losses together, in fp16: its steps stay finite and it learns."""
import json
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu


def test_the_step_learns_in_fp16():
    r = subprocess.run([sys.executable, "-m", "paper_2511_13645_amd.entity_step", "--nodes", "3000", "--dim", "64", "--batch", "256",
                        "--slots", "8", "--steps", "30", "--dtype", "f16"], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    line = json.loads(r.stdout.strip().splitlines()[-1])
    assert line["last_loss"] < line["first_loss"]
