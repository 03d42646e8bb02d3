"""The search for a workgroup's tile in packed sequences (csrc/grkan_packed.h), run on the host lane by lane: rising offsets give every tile once and the longest
walks first; falling ones nothing outside of the buffer and its places, though tiles may be nobody's then."""
import shutil
import subprocess
from pathlib import Path

import pytest

SOURCE = Path(__file__).resolve().parent / "native" / "segments_selftest.cpp"


def test_every_tile_has_one_workgroup(tmp_path):
    compiler = shutil.which("g++")
    if compiler is None:
        pytest.skip("no g++ on this machine")
    program = tmp_path / "segments"
    built = subprocess.run([compiler, "-std=c++17", "-O2", "-Wall", "-Wno-unknown-pragmas", str(SOURCE), "-o", str(program)], capture_output=True, text=True)
    assert built.returncode == 0, built.stderr
    found = subprocess.run([str(program)], capture_output=True, text=True, timeout=120)
    assert found.returncode == 0 and found.stdout == "every tile once\n", found.stdout[:4000]
