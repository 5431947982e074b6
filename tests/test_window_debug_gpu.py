"""The tests of rotary positions with several axes and of windowed attention under the bounds-checked library, with canary
words around what the binding allocates."""
import os
import subprocess
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu

ROOT = Path(__file__).resolve().parent.parent


def test_windowed_attention_under_the_bounds_checked_library():
    from paper_2407_20485_b200 import build

    build.build(debug=True)
    env = dict(os.environ, A2SF_LIBRARY="debug", A2SF_GUARDS="1")
    cmd = [sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider", "tests/test_window_gpu.py", "tests/test_rotary_axes_gpu.py"]
    r = subprocess.run(cmd, cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    tail = r.stdout[-3000:] + r.stderr[-2000:]
    assert r.returncode == 0, tail
    line = [x for x in r.stdout.splitlines() if x.startswith("[debug sweep]")]
    assert line, tail
    from conftest import report_line

    report_line(line[0] + " (windowed attention)")
    assert " 0 index violations" in line[0]
    assert int(line[0].split()[2]) >= 150, line[0]
