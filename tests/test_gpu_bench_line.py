"""bench.py's line on standard output stays short enough to be read whole: what is long goes to standard error."""
import json
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_one_short_line_and_the_details_apart():
    r = subprocess.run([sys.executable, os.path.join(ROOT, "bench.py"), "--config", "3", "--clients", "2", "--steps", "2", "--warmup", "3",
                        "--no-table", "--no-cpu-baseline"], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    lines = r.stdout.splitlines()
    assert len(lines) == 1 and len(lines[0]) < 3000
    d = json.loads(lines[0])
    for key in ("metric", "value", "unit", "n_gpus", "steps", "warmup", "ms_per_step", "higher_is_better", "scaling", "vs_baseline", "dtype",
                "data", "config", "gpu_launches", "roofline", "clocks", "e2e"):
        assert key in d
    assert d["value"] > 0 and d["e2e"]["value"] > 0 and d["gpu_launches"] > 0
    more = json.loads([l for l in r.stderr.splitlines() if l.startswith('{"details"')][-1])["details"]
    assert "pack" in more["kernels"] and more["per_config"][0]["workload"] == d["config"]["workload"]
