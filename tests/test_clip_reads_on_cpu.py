"""What gradient norms and clipping read and write, followed on the CPU: every thread of every
launch runs under AddressSanitizer on buffers of just the bytes that cpdp.h lets a call
touch."""
import math
import os
import random
import subprocess

import pytest

import on_cpu
from paper_2607_21224_amd import build

pytestmark = pytest.mark.skipif(not on_cpu.available(), reason="needs ROCm's clang")


@pytest.fixture(scope="module")
def good(tmp_path_factory):
    folder = str(tmp_path_factory.mktemp("clip"))
    here, csrc = os.path.join(on_cpu.NATIVE, "on_cpu_clip"), os.path.join(build.PKG, "csrc")
    exe = os.path.join(folder, "clip_calls")
    sources = [os.path.join(csrc, s) for s in build.CLIP_SOURCES]
    r = subprocess.run([on_cpu.CLANG, *on_cpu.FLAGS, "-O1", "-I", here, "-I",
                        os.path.join(build.ROOT, "include"), "-I", csrc, "-no-pie", "-x", "c++",
                        *sources, os.path.join(here, "clip_calls.cpp"), "-o", exe, "-lstdc++",
                        "-lm"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(lines):
        lines = [" ".join(map(str, c)) for c in lines]
        r = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True)
        got = r.stdout.splitlines()
        assert r.returncode == 0, (lines[len(got)], r.stderr[-4000:])
        assert got == ["0"] * len(lines)
    return run


@pytest.mark.parametrize("bf16", [0, 1])
@pytest.mark.parametrize("mean", [0, 1])
def test_rows(good, bf16, mean):
    sizes = [0, 1, 2, 3, 4, 5, 7, 8, 9, 255, 256, 257, 511, 1023, 1025, 2047, 4097, 8191, 8200,
             16390, 70001]
    good([("flat", W, P, bf16, mean, clip) for P in sizes for W in (1, 3) for clip in (0, 1)])
    # more replicas than parts, and rows past what is clipped in small blocks
    good([("flat", 2100, 5, bf16, mean, 1), ("flat", 40, 5003, bf16, mean, 1),
          ("flat", 9, (1 << 22) + 13, bf16, mean, 1)])


@pytest.mark.parametrize("mean", [0, 1])
def test_tensors(good, mean):
    rng = random.Random(4)
    cases = [[1], [0, 5, 0, 257, 1], [64, 64, 4096, 64, 7, 1000], [1] * 300, [0], [0, 0, 2, 0],
             [300000, 3, 0, 70001]]
    cases += [[int(math.exp(rng.uniform(0, 9))) for _ in range(rng.randint(1, 40))]
              for _ in range(12)]
    good([("plan", W, mean, clip, *c) for c in cases for W in (1, 4) for clip in (0, 1)])
    good([("plan", 5, mean, 1, 3500001, 5, 64, 0, 100, 9)])
