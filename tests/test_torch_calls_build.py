"""The extension that marshals torch tensors: the rest of the package does without it, and one of another torch is not loaded."""
import subprocess
import sys
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent


def python(code):
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=600, cwd=ROOT)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
    return r.stdout


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2407_20485_b200 import build

    build.build()


def test_without_the_extension_only_its_own_calls_are_missing(tmp_path):
    python(f"""
from pathlib import Path
from paper_2407_20485_b200 import build
build.calls_path = lambda: Path({str(tmp_path / 'none.so')!r})
import torch
from paper_2407_20485_b200 import binding as a2sf
p = a2sf.make_params(1, 2, 64, torch.float32, 8, 2, 0.5)
assert a2sf.a2sf_kernel_launch_count() == 0
plan = a2sf.a2sf_rotary_plan_init(64)
for call in (lambda: a2sf.a2sf_rotary(plan, torch.zeros(1, 1, 1, 64)), lambda: a2sf.PagedCache(1, 1, 64, torch.float32, 16, 1, 1, device='cpu')):
    try:
        call()
    except ImportError as e:
        assert 'paper_2407_20485_b200.build' in str(e), e
    else:
        raise AssertionError('no ImportError')
""")


def test_an_extension_of_another_torch_is_not_taken_for_this_one():
    """What the build writes and the binding loads is named after the interpreter and the torch that it was made for."""
    out = python("""
import torch
from paper_2407_20485_b200 import build
here = build.calls_path()
torch.__version__ = '9.9.9+other'
there = build.calls_path()
assert here != there and here.suffix == there.suffix == '.so'
assert here.exists() and not there.exists()
print('ok')
""")
    assert "ok" in out


def test_the_library_builds_without_torch():
    python("""
import sys
sys.modules['torch'] = None                     # import torch fails
from paper_2407_20485_b200 import build
assert build.build() == build.LIB_PATH
""")
