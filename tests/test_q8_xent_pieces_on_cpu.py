"""Gradients of the loss in pieces that the laid-out weights bound, followed on the CPU under
AddressSanitizer as test_q8_xent_reads_on_cpu.py follows the others."""
from concurrent.futures import ThreadPoolExecutor

import pytest

import on_cpu
import xent_on_cpu
import xent_sizes

pytestmark = pytest.mark.skipif(not on_cpu.available(), reason="needs ROCm's clang")


def test_several_pieces(tmp_path):
    exe = xent_on_cpu.compile_calls(str(tmp_path), "-O1")
    lines = [" ".join(map(str, ("xent_bwd", *s, *t)))
             for i, s in enumerate(xent_sizes.WEIGHTS)
             for t in (xent_sizes.TYPES[i % 4], xent_sizes.ALONE[i % 4])]
    with ThreadPoolExecutor(3) as pool:
        for line, got in zip(lines, pool.map(lambda c: on_cpu.run(exe, "run", [c]), lines)):
            (status, kernels), = got
            assert status == 0 and len(kernels) >= 2 and "large" not in kernels, line
