"""bench.py with the layer between its projections: what the line says about the step, and what it checks."""
import json
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _line(*args):
    run = subprocess.run([sys.executable, os.path.join(ROOT, "bench.py"), "--workload", "layer16", "--steps", "2", "--warmup", "3", "--cpu-sample", "32", *args],
                         check=True, capture_output=True, text=True, cwd=ROOT)
    return json.loads(run.stdout.strip().splitlines()[-1])


def test_the_step_from_tokens_is_described_as_what_it_is():
    line = _line("--from-tokens", "128", "--batch", "1x16x80", "--no-e2e")
    assert line["roofline"] is None                                  # eleven kernels, no single bound
    assert "10 x ttc_linear" in line["config"]["kernel"] and "y" in line["config"]["outputs"]
    assert line["launches_per_step"] == 11                           # none of them needs a second launch
    errs = line["cpu_baseline"]["parity_rows_rel_norm"]
    assert len(errs) == 11 and errs["y"] > 0
    # rows of odd width are copied first, in launches that are not counted
    assert _line("--from-tokens", "1101", "--batch", "1x16x40", "--no-e2e")["launches_per_step"] is None
    plain = _line("--batch", "1x16x80", "--no-e2e")
    assert plain["roofline"]["kernel"] == plain["config"]["kernel"] == "ttc_layer" and plain["launches_per_step"] >= 1
