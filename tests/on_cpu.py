"""Builds and drives tests/native/on_cpu/q8_calls: the 8-bit path's kernels and launchers
compiled for the host."""
import os
import shutil
import subprocess

from paper_2607_21224_amd import build

NATIVE = os.path.join(build.ROOT, "tests", "native")
CLANG = os.path.join(os.path.dirname(os.path.dirname(build.HIPCC)), "llvm", "bin", "clang++")
FLAGS = ["-std=c++17", "-g1", "-fno-pie", "-fno-omit-frame-pointer",
         "-fsanitize=address,alignment", "-fno-sanitize-recover=all"]


def available():
    return shutil.which(CLANG) is not None


def compile_calls(folder, optimise="-O0"):
    """The program, built in `folder`; as it is, a load whose result nothing uses is made all
    the same, optimised, calls of some size run in a second."""
    csrc = os.path.join(build.PKG, "csrc")
    sources = [os.path.join(csrc, s) for s in build.Q8_SOURCES]
    sources.append(os.path.join(NATIVE, "on_cpu", "q8_calls.cpp"))
    include = ["-I", os.path.join(NATIVE, "on_cpu"), "-I", os.path.join(build.ROOT, "include"),
               "-I", csrc]
    jobs, objects = [], []
    for s in sources:
        objects.append(os.path.join(folder, os.path.basename(s) + ".o"))
        jobs.append(subprocess.Popen([CLANG, *FLAGS, optimise, *include, "-x", "c++", "-c", s, "-o",
                                      objects[-1]], stdout=subprocess.PIPE,
                                     stderr=subprocess.STDOUT, text=True))
    for j in jobs:
        text = j.communicate()[0]
        assert j.returncode == 0, text
    exe = os.path.join(folder, "q8_calls")
    r = subprocess.run([CLANG, "-fsanitize=address,alignment", "-no-pie", "-o", exe, *objects],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return exe


def run(exe, mode, calls):
    """The answer to each call: its status and the kernels it launched (addresses)."""
    r = subprocess.run([exe, mode], input="\n".join(calls) + "\n", capture_output=True, text=True)
    lines = r.stdout.splitlines()
    assert r.returncode == 0, (calls[len(lines)], r.stderr[-4000:])
    assert len(lines) == len(calls)
    return [(int(w[0]), w[1:]) for w in map(str.split, lines)]
