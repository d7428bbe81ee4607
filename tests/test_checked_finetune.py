"""The fine-tuning operators in the checked build (internal invariants asserted into the
status word): clean status words, and the same bits as the normal build."""
import os
import subprocess
import sys

import numpy as np
import pytest

from paper_2608_09703_gb300 import build as mbuild

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def run_child(path, checked):
    env = dict(os.environ, MLS_CHECKED="1" if checked else "0")
    env["PYTHONPATH"] = ROOT + os.pathsep + env.get("PYTHONPATH", "")
    r = subprocess.run([sys.executable, os.path.join(ROOT, "tests", "checked_finetune_run.py"), path],
                       env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout + r.stderr
    return dict(np.load(path))


def test_checked_build_is_clean_and_identical(tmp_path):
    mbuild.build()
    mbuild.build(checked=True)
    normal = run_child(str(tmp_path / "normal.npz"), checked=False)
    checked = run_child(str(tmp_path / "checked.npz"), checked=True)
    assert set(normal) == set(checked)
    for k in checked:
        if k.startswith("status"):
            assert int(checked[k]) == 0 and int(normal[k]) == 0, k
        else:
            assert np.array_equal(checked[k], normal[k]), k
