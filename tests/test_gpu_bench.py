"""The benchmark's options run as they are documented."""
import json
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("options", [[], ["--kv", "int4"], ["--policy", "window"]], ids=["bf16", "int4", "window"])
def test_mixed_lengths(options):
    if "int4" in options:
        options = options + ["--workload", "llama", "--layers", "1"]
    else:
        options = options + ["--workload", "tiny"]
    run = subprocess.run([sys.executable, "bench.py", "--mixed-lengths", "--steps", "4", "--warmup", "3", "--no-cpu-baseline"] + options,
                         cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]
    line = json.loads(run.stdout.strip().splitlines()[-1])
    assert line["steps"] == 4 and line["ms_per_step"] > 0 and line["e2e"]["value"] > 0
