"""Which kernels of the 8-bit path the calls of q8_sizes.py take: each that is compiled into
it runs, so that the GPU tests compare it and none is kept that no call reaches; and that
all they read and write in these calls is in range."""
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

import on_cpu
import q8_sizes

pytestmark = pytest.mark.skipif(not on_cpu.available(), reason="needs ROCm's clang")


def kernels_of(exe):
    """{address: name} of the kernels in the program."""
    r = subprocess.run(["nm", "-C", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    out = {}
    for line in r.stdout.splitlines():
        address, kind, name = line.split(" ", 2) if line[:1] != " " else ("", "", "")
        name = name.replace("(anonymous namespace)::", "").replace("(cpdp::q8::Act)", "")
        m = re.match(r"(?:void )?cpdp::q8::([a-z0-9_]+_kernel)(<[^()]*>)?\([^{]*\)$", name)
        if kind in ("t", "T", "w", "W") and m and not m[1].startswith("launch"):
            out[address.lstrip("0")] = m[1] + (m[2] or "")
    return out


@pytest.fixture(scope="module")
def launched(tmp_path_factory):
    """{kernel: the calls that take it}, with all kernels there are."""
    exe = on_cpu.compile_calls(str(tmp_path_factory.mktemp("on_cpu")))
    names = kernels_of(exe)
    assert len(set(names.values())) > 150
    out = {n: [] for n in names.values()}
    calls = list(q8_sizes.calls())
    for call, (status, kernels) in zip(
            calls, on_cpu.run(exe, "note", [" ".join(map(str, c)) for c in calls])):
        assert status == 0, call
        for k in kernels:
            out[names[k]].append(call)
    return out


def test_every_kernel_is_reached(launched):
    left = sorted(n for n, calls in launched.items() if not calls)
    assert not left, "\n".join(left)


def test_all_that_they_touch_is_in_range(tmp_path):
    """(test_q8_reads_on_cpu.py goes through more sizes, smaller ones)"""
    exe = on_cpu.compile_calls(str(tmp_path), "-O1")
    calls = [" ".join(map(str, c)) for c in q8_sizes.calls()]
    with ThreadPoolExecutor(8) as pool:
        parts = [calls[i::32] for i in range(32)]
        for part, answers in zip(parts, pool.map(lambda p: on_cpu.run(exe, "run", p), parts)):
            for call, (status, kernels) in zip(part, answers):
                assert status == 0 and "large" not in kernels, call
