"""The kernels for attention to states and for norms with rotation may start under the kernel that writes their inputs, and read those behind its end.  The read-only path (`__ldg`, ld.global.nc, or what
`const ... __restrict__` permits the compiler) is for memory that nothing writes while a kernel is there: none of them may use it."""
import re

import pytest

from paper_2603_06738_b200 import build

FILES = sorted([*build.CSRC.glob("rib_cross*"), build.CSRC / "rib_rope.cu"])


def code(path):
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", path.read_text(), flags=re.S)


def test_the_files_are_there():
    assert len(FILES) == 7 and all("launch_overtaking" in code(f) or f.suffix == ".cuh" for f in FILES)


@pytest.mark.parametrize("path", FILES, ids=lambda f: f.name)
def test_no_read_only_path(path):
    for word in ("__restrict__", "__restrict", "__ldg", "ld.global.nc", "ld.const"):
        assert word not in code(path), word
