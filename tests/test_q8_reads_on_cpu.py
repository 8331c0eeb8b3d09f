"""What the 8-bit path's kernels read and write, followed on the CPU: every thread of every
launch runs under AddressSanitizer on buffers of just the bytes that cpdp_q8.h lets a call
touch, what lies between two rows poisoned.  Sizes are ragged ones around the kernels'
pieces, steps and tiles, and random ones."""
import math
import random

import pytest

import on_cpu

pytestmark = pytest.mark.skipif(not on_cpu.available(), reason="needs ROCm's clang")

F32, BF16, NONE = 0, 1, -1
TYPES = [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)]
# both sides of what a row's shape depends on
WIDTHS = [1, 7, 8, 9, 511, 512, 513, 1024, 1025, 2047, 2049, 4096, 4103, 8192, 8195, 16385, 32769]


@pytest.fixture(scope="module")
def calls(tmp_path_factory):
    exe = on_cpu.compile_calls(str(tmp_path_factory.mktemp("on_cpu")))
    return lambda lines: on_cpu.run(exe, "run", [" ".join(map(str, c)) for c in lines])


def good(calls, lines):
    for line, (status, kernels) in zip(lines, calls(lines)):
        assert status == 0 and kernels and "large" not in kernels, (line, status, kernels)


def sizes(seed, count, *most):
    """Tuples of sizes from 1, spread over their logarithm."""
    rng = random.Random(seed)
    return [tuple(max(1, round(math.exp(rng.uniform(0, math.log(m))))) for m in most)
            for _ in range(count)]


def test_rows_and_values(calls):
    good(calls, [("rows", T, D, x, y) for D in WIDTHS for T in (1, 5) for x in (F32, BF16)
                 for y in (NONE, F32, BF16)] +
         [("values", T, D, y) for D in WIDTHS for T in (1, 5) for y in (F32, BF16)] +
         [("rows", 4099, D, BF16, NONE) for D in (700, 1300)])


def test_norm(calls):
    good(calls, [("norm", T, D, a, w, r, y) for D in WIDTHS for T in (1, 5) for a, w in TYPES
                 for r, y in ((0, NONE), (1, BF16))] +
         [("norm", 4099, D, F32, F32, 1, BF16) for D in (700, 1300)])


def test_norm_bwd(calls):
    good(calls, [("norm_bwd", T, D, a, w, r, w) for D in WIDTHS for T in (1, 5, 70)
                 for a, w in TYPES for r in (0, 1)] +
         [("norm_bwd", T, D, BF16, F32, 1, F32)
          for T, D in ((1576, 384), (2051, 515), (1030, 1031), (1029, 4095))])


def test_activations(calls):
    good(calls, [("act", k, T, F, a, y, c) for k in (0, 1) for F in WIDTHS for T in (1, 5)
                 for a in (F32, BF16) for y, c in ((NONE, 0), (BF16, 1))] +
         [("act_bwd", k, T, F, a) for k in (0, 1) for F in WIDTHS for T in (1, 5)
          for a in (F32, BF16)])


def test_products(calls):
    good(calls, [("product", *s, y) for s in sizes(1, 60, 200, 200, 1500) for y in (F32, BF16)] +
         [("product", M, N, K, F32) for M in (1, 16, 17, 33, 64, 65) for N in (1, 17, 130)
          for K in (1, 15, 16, 17, 127, 128, 129, 300)])


@pytest.mark.parametrize("op", ["grad_input", "grad_weight"])
def test_gradients(calls, op):
    good(calls, [(op, *s, *t) for s in sizes(2, 40, 300, 400, 300) for t in TYPES])


# Lane groups of the last of 32 values of the sum that begin past its end have no scales.
@pytest.mark.parametrize("T", [1, 17, 32])
def test_input_gradients_of_few_tokens(calls, T):
    good(calls, [("grad_input", T, N, K, *t) for N in range(1, 129) for K in (1, 130)
                 for t in ((F32, F32), (BF16, BF16))] +
         [("grad_input", T, N, 9, *t) for N in (225, 1000, 1153) for t in TYPES])


@pytest.mark.parametrize("T", [1, 31, 33, 64])
def test_weight_gradients_of_few_tokens(calls, T):
    good(calls, [("grad_weight", T, N, K, *t) for N in (1, 2, 31, 33, 257)
                 for K in (1, 3, 64, 65, 131) for t in TYPES])
