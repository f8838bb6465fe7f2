"""The host-only calls need numpy alone: they run in a process that has no torch."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
import sys
sys.modules["torch"] = None                       # an import of it fails
import numpy as np
from paper_2503_22796_amd import binding as B
st, items, _ = B.difa_worklist_build(1, 2, [0, 1], [0, 40], 16, 300, 128, 64)
assert st == B.DIFA_OK and len(items) > 0
st, segs, wg_begin, _, _ = B.difa_schedule_build(items, 4, 1)
assert st == B.DIFA_OK and wg_begin[-1] == len(segs) > 0
st, choice, _, _ = B.difa_plan_solve(np.array([[0.1, 0.9], [0.8, 0.2]]), np.array([1.0, 2.0]), 4.0, 10.0, 2.0)
assert st == B.DIFA_OK and list(choice) == [0, 0]
print("ran")
"""


def test_worklists_schedules_and_plans_without_torch():
    got = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert got.returncode == 0 and got.stdout.strip() == "ran", got.stderr
