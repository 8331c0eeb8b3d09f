"""The validation layer of the 8-bit path, built for the host with AddressSanitizer
and UndefinedBehaviorSanitizer and driven through valid and invalid calls."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NATIVE = os.path.join(ROOT, "tests", "native")
CSRC = os.path.join(ROOT, "paper_2607_21224_amd", "csrc")
SAN = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer",
       "-g", "-O1"]


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_validation_under_sanitizers(tmp_path):
    exe = str(tmp_path / "q8_driver")
    cmd = ["g++", "-std=c++17", "-Wall", *SAN, "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           os.path.join(CSRC, "q8_api.cpp"), os.path.join(NATIVE, "q8_stub.cpp"),
           os.path.join(NATIVE, "q8_driver.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "OK", r.stdout + r.stderr
