"""Launch sizes of the language-model operators, checked on the host: the same header the library is compiled from, built with the host
compiler."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host C++ compiler")
def test_launches_hold_what_a_launch_may(tmp_path):
    exe = str(tmp_path / "lm_launch_check")
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-Wall", "-o", exe, os.path.join(HERE, "lm_launch_check.cpp")])
    r = subprocess.run([exe], stdout=subprocess.PIPE, text=True)
    assert r.returncode == 0 and int(r.stdout) > 8000, r.stdout
