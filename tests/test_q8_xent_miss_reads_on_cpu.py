"""What the calls of the loss with a token's miss read and write, followed on the CPU under
AddressSanitizer as test_q8_xent_reads_on_cpu.py follows the others: every kernel that the sizes
of the GPU tests take."""
from concurrent.futures import ThreadPoolExecutor

import pytest

import on_cpu
import xent_on_cpu
import xent_sizes

pytestmark = pytest.mark.skipif(not on_cpu.available(), reason="needs ROCm's clang")

BWD = [*xent_sizes.TYPES, *xent_sizes.ALONE]


def test_the_gpu_tests_sizes(tmp_path):
    exe = xent_on_cpu.compile_calls(str(tmp_path), "-O1", calls="xent_miss_calls.cpp")
    sizes = xent_sizes.SMALL + xent_sizes.MIDDLE
    calls = [("xent_miss", *s) for s in sizes]
    calls += [("xent_miss_bwd", *s, *BWD[i % len(BWD)]) for i, s in enumerate(sizes)]
    lines = [" ".join(map(str, c)) for c in calls]
    parts = [lines[i::16] for i in range(16)]
    with ThreadPoolExecutor(8) as pool:
        for part, got in zip(parts, pool.map(lambda p: on_cpu.run(exe, "run", p), parts)):
            for line, (status, kernels) in zip(part, got):
                assert status == 0 and kernels and "large" not in kernels, line
