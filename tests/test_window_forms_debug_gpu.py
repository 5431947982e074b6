"""Every form of the windowed attention under the bounds-checked library, and that the forms check their indexes there."""
import os
import re
import subprocess
import sys
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
FORM_TESTS = ["tests/test_window_nan_gpu.py", "tests/test_window_precision_gpu.py", "tests/test_window_chunk_kernel_gpu.py"]


def test_every_kernel_of_few_rows_checks_its_own_indexes():
    text = (ROOT / "paper_2407_20485_b200" / "csrc" / "paged_attn_few.cu").read_text()
    found = list(re.finditer(r"__global__[^;{]*?(paged_\w+)\([^;{]*?\)\n\{\n", text))
    assert len(found) == text.count("__global__")
    for m in found:
        assert "A2SF_IN_RANGE" in text[m.end():text.index("\n}\n", m.end())], m.group(1)


@pytest.mark.gpu
def test_all_forms_under_the_bounds_checked_library():
    from paper_2407_20485_b200 import build

    build.build(debug=True)
    env = dict(os.environ, A2SF_LIBRARY="debug", A2SF_GUARDS="1")
    cmd = [sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider", *FORM_TESTS]
    r = subprocess.run(cmd, cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    tail = r.stdout[-3000:] + r.stderr[-2000:]
    assert r.returncode == 0, tail
    line = [x for x in r.stdout.splitlines() if x.startswith("[debug sweep]")]
    assert line, tail
    from conftest import report_line

    report_line(line[0] + " (forms of the windowed attention)")
    assert " 0 index violations" in line[0]
    assert int(line[0].split()[2]) >= 50, line[0]
