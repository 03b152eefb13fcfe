"""The library and torch have to share one HIP runtime, whichever is imported first: with two in a process the library's finds no device."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("first,second", [("paper_2410_17043_amd", "torch"), ("torch", "paper_2410_17043_amd")])
def test_one_hip_runtime_is_loaded(first, second):
    code = ("import %s, %s\nprint(len({l.split()[-1] for l in open('/proc/self/maps') if 'libamdhip64' in l}),"
            " sum('libaurora_moe' in l for l in open('/proc/self/maps')) > 0)") % (first, second)
    out = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, check=True, timeout=300).stdout
    assert out.split() == ["1", "True"]
