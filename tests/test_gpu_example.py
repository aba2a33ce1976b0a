"""The example runs the token operators together: what it learns is learned."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_distill_example(gpu):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import distill
    finally:
        sys.path.pop(0)
    lines = []
    r = distill.run(steps=300, report=lines.append)
    # untrained: near the uniform distribution's log 5003 = 8.52; the text's own
    # conditional entropy is 1.75 bits, 1.21 nats
    assert -9.5 < r["start"][0] < -8.0
    assert -3.0 < r["teacher"][0] < -1.2
    assert r["student"][0] > -5.0 and r["loss"] < r["first_loss"] / 3
    assert len(r["said"][0]) == len(r["said"][1]) == 8 and len(lines) == 14
    again = distill.run(steps=2, report=None)
    assert again["start"] == r["start"]


def test_distill_example_command(gpu):
    out = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "distill.py"), "--vocabulary",
                          "307", "--batch", "64", "--steps", "50", "--top", "5"], check=True,
                         capture_output=True, text=True, timeout=100).stdout
    assert "student step   50" in out and "after token 1" in out and "nan" not in out
