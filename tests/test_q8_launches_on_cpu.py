"""Launches of the 8-bit path at the ends of the sizes that it takes, on the CPU: each holds
fewer than 2^32 work items in a direction of its grid, which is all the runtime takes."""
import pytest

import on_cpu

pytestmark = pytest.mark.skipif(not on_cpu.available(), reason="needs ROCm's clang")

F32, BF16, NONE = 0, 1, -1
ROWS, COLS = (1 << 31) - 9, (1 << 28) - 64  # the most rows, about the longest rows


@pytest.fixture(scope="module")
def calls(tmp_path_factory):
    exe = on_cpu.compile_calls(str(tmp_path_factory.mktemp("on_cpu")))
    return lambda lines: on_cpu.run(exe, "note", [" ".join(map(str, c)) for c in lines])


@pytest.mark.parametrize("line", [
    ("rows", 1, COLS, BF16, NONE), ("rows", ROWS, 64, F32, NONE), ("rows", ROWS, 513, BF16, NONE),
    ("values", 40, COLS, BF16), ("values", ROWS, 8, F32),
    ("norm", 1, COLS, BF16, F32, 1, BF16), ("norm", ROWS, 64, F32, F32, 0, NONE),
    ("norm_bwd", 1, (1 << 27) + 8, BF16, F32, 0, F32), ("norm_bwd", 1, COLS, F32, F32, 1, BF16),
    ("norm_bwd", ROWS, 8, BF16, BF16, 1, F32),
    ("act", 1, 1, COLS, BF16, NONE, 1), ("act", 0, ROWS, 64, BF16, NONE, 0),
    ("act_bwd", 1, 40, COLS, BF16), ("act_bwd", 0, ROWS, 8, F32),
    ("product", (1 << 31) - 1024, 8, 64, BF16), ("product", 64, COLS, 1000, F32),
    ("product", 65, COLS, 64, BF16)])
def test_work_items(calls, line):
    (status, kernels), = calls([line])
    assert status == 0 and kernels and "large" not in kernels, (status, kernels)
