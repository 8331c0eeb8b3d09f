"""What the loss' kernels read and write, followed on the CPU: every thread of every launch
runs under AddressSanitizer on buffers of just the bytes that cpdp_q8.h lets a call touch."""
from concurrent.futures import ThreadPoolExecutor

import pytest

import on_cpu
import xent_on_cpu
import xent_sizes
from test_q8_reads_on_cpu import sizes

pytestmark = pytest.mark.skipif(not on_cpu.available(), reason="needs ROCm's clang")

BWD = [*xent_sizes.TYPES, *xent_sizes.ALONE]


@pytest.fixture(scope="module")
def good(tmp_path_factory):
    exe = xent_on_cpu.compile_calls(str(tmp_path_factory.mktemp("on_cpu")), "-O1")

    def run(lines):
        lines = [" ".join(map(str, c)) for c in lines]
        parts = [lines[i::32] for i in range(32) if lines[i::32]]
        with ThreadPoolExecutor(8) as pool:
            for part, got in zip(parts, pool.map(lambda p: on_cpu.run(exe, "run", p), parts)):
                for line, (status, kernels) in zip(part, got):
                    assert status == 0 and kernels and "large" not in kernels, line
    return run


@pytest.mark.parametrize("seed", range(3))
def test_random_sizes(good, seed):
    some = sizes(seed, 40, 300, 700, 300)
    good([("xent", *s) for s in some])
    good([("xent_bwd", *s, *BWD[i % len(BWD)]) for i, s in enumerate(some)])


def test_the_gpu_tests_sizes(good):
    good([("xent", *s) for s in xent_sizes.SMALL + xent_sizes.MIDDLE])
    good([("xent_bwd", *s, *t) for s in xent_sizes.SMALL for t in BWD])
    good([("xent_bwd", *s, *t) for s in xent_sizes.MIDDLE for t in xent_sizes.TYPES])


def test_several_pieces(good):
    good([("xent", *s) for s in xent_sizes.LARGE])
    good([("xent_bwd", *s, *xent_sizes.TYPES[i % 4]) for i, s in enumerate(xent_sizes.LARGE)])
