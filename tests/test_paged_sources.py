"""The order that programmatic launches rest on, read from the sources: no GPU."""
import re
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2407_20485_b200" / "csrc"


def kernels():
    for path in sorted([*CSRC.glob("paged_*.cu"), CSRC / "rotary.cu"]):
        text = path.read_text()
        for m in re.finditer(r"__global__[^;{]*?((?:paged|rotary)_\w+)\([^;{]*?\)\n\{\n", text):
            yield pytest.param(text[m.end():text.index("\n}\n", m.end())], id=f"{path.stem}-{m.group(1)}")


@pytest.mark.parametrize("body", list(kernels()))
def test_followers_may_start_only_behind_a_wait(body):
    """Every kernel waits for its predecessors; the followers' start is allowed, where it is allowed early, after a wait."""
    assert "dependency_wait();" in body
    if "dependents_may_start();" in body:
        assert body.index("dependency_wait();") < body.index("dependents_may_start();")


def test_the_kernels_are_found():
    found = sum((path.read_text().count("__global__") for path in [*CSRC.glob("paged_*.cu"), CSRC / "rotary.cu"]))
    assert len(list(kernels())) == found
