"""The order of loads, waits, barriers and reads in the causal attention kernel whose wavefronts take turns (csrc/grkan_turns.h), run on the host as the
kernel runs it: whatever is read has been waited for by all that loaded a part of it, in front of a barrier before the read, and no place is loaded
to before all have read it."""
import shutil
import subprocess
from pathlib import Path

import pytest

SOURCE = Path(__file__).resolve().parent / "native" / "turns_selftest.cpp"


def test_what_is_read_has_been_waited_for(tmp_path):
    compiler = shutil.which("g++")
    if compiler is None:
        pytest.skip("no g++ on this machine")
    program = tmp_path / "turns"
    built = subprocess.run([compiler, "-std=c++17", "-O1", "-Wall", "-Wno-unknown-pragmas", str(SOURCE), "-o", str(program)], capture_output=True, text=True)
    assert built.returncode == 0, built.stderr
    found = subprocess.run([str(program)], capture_output=True, text=True, timeout=60)
    assert found.returncode == 0 and found.stdout == "in order\n", found.stdout[:4000]
