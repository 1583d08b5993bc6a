"""How the logits' copy shares its vocabulary out, checked on the host: the same header the library is compiled from, built with the host compiler."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host C++ compiler")
def test_vocabularies_up_to_the_largest(tmp_path):
    exe = str(tmp_path / "logits_parts_check")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=signed-integer-overflow", "-fno-sanitize-recover=all", "-o", exe, os.path.join(HERE, "logits_parts_check.cpp")])
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0 and int(r.stdout) > 1000, r.stdout
