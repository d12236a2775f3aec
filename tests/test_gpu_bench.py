"""bench.py with few steps: fewer than a launch of several rounds takes."""
import json
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("steps", [1, 3])
def test_few_steps_have_a_line(steps):
    cmd = [sys.executable, "bench.py", "--p", "600000", "--steps", str(steps), "--warmup", "1", "--no-cpu-baseline"]
    res = subprocess.run(cmd, cwd=ROOT, capture_output=True, text=True, timeout=100)
    assert res.returncode == 0, res.stderr[-2000:]
    line = [json.loads(x) for x in res.stdout.splitlines() if x.startswith("{")][-1]
    assert line["steps"] == steps and line["warmup"] == 1 and line["value"] > 0
    roof = line["roofline"]
    assert roof["launches"] == steps and 0 < roof["frac"] and roof["avg_kernel_ms"] > 0 and roof["bytes_per_launch"] > 0
