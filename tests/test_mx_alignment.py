"""Products of 4-bit layers read rows of X whose ends lie anywhere: where those loads begin, on the host, over all ends of rows."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_loads_of_16_bytes_begin_at_words(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    exe = str(tmp_path / "mx_alignment")
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-o", exe, os.path.join(ROOT, "tests", "native", "mx_alignment.cpp")], check=True, timeout=120)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and " 0 failures" in run.stdout, run.stdout
