"""Builds tests/native/on_cpu/xent_calls: the loss' kernels and launchers, and those of the
8-bit path that it calls, compiled for the host."""
import os
import subprocess

import on_cpu
from paper_2607_21224_amd import build

# the kernels of its own units
NAMES = ("xent", "head")


def compile_calls(folder, optimise="-O0", sources=None, calls="xent_calls.cpp"):
    csrc = os.path.join(build.PKG, "csrc")
    paths = [os.path.join(csrc, s) for s in sources or build.Q8_SOURCES + build.XENT_SOURCES]
    paths.append(os.path.join(on_cpu.NATIVE, "on_cpu", calls))
    include = ["-I", os.path.join(on_cpu.NATIVE, "on_cpu_xent"), "-I",
               os.path.join(on_cpu.NATIVE, "on_cpu"), "-I",
               os.path.join(build.ROOT, "include"), "-I", csrc]
    jobs, objects = [], []
    for p in paths:
        objects.append(os.path.join(folder, os.path.basename(p) + ".o"))
        jobs.append(subprocess.Popen([on_cpu.CLANG, *on_cpu.FLAGS, optimise, *include, "-x", "c++",
                                      "-c", p, "-o", objects[-1]], stdout=subprocess.PIPE,
                                     stderr=subprocess.STDOUT, text=True))
    for j in jobs:
        text = j.communicate()[0]
        assert j.returncode == 0, text
    exe = os.path.join(folder, "xent_calls")
    r = subprocess.run([on_cpu.CLANG, "-fsanitize=address,alignment", "-no-pie", "-o", exe,
                        *objects], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return exe
