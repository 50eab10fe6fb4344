"""`python __graft_entry__.py --smoke`, the file as a program: what it calls has to be defined when it runs."""
import ast
import subprocess
import sys
from pathlib import Path

import pytest

ENTRY = Path(__file__).resolve().parent.parent / "__graft_entry__.py"


def test_the_program_part_comes_last():
    body = ast.parse(ENTRY.read_text()).body
    programs = [i for i, node in enumerate(body) if isinstance(node, ast.If) and "__name__" in ast.dump(node.test)]
    assert programs == [len(body) - 1]


# The library as it is built: a program that compiles it anew would take the files away under the tests that run.
PROGRAM = """
import runpy, sys
from paper_2603_06738_b200 import build
from oracle import rib_oracle
compile_oracle = rib_oracle.build
build.build = lambda force=False, verbose=False: build.LIB
rib_oracle.build = lambda force=False: compile_oracle()
sys.argv = [sys.argv[1], "--smoke"]
runpy.run_path(sys.argv[0], run_name="__main__")
"""


@pytest.mark.gpu
def test_the_program_runs():
    run = subprocess.run([sys.executable, "-c", PROGRAM, str(ENTRY)], cwd=ENTRY.parent, capture_output=True, text=True, timeout=600)
    assert run.returncode == 0, run.stderr[-2000:]
    assert "attention to 300 states" in run.stdout
