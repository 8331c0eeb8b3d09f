"""GELU of rows whose results are all small because their inputs are far below zero: a row
has a scale of its own, so there is nothing large beside which their error would vanish.

Tolerance, u = 2^-24, relative to the row's largest result: the upper tail's argument
-g / sqrt(2) takes two roundings, which its value has (g^2 + 1)-fold; the library's function
is taken to be good to 16 units in the last place (32 u), and there are a few products.
Above -2 the results come of 1 + erf: |g| u and a few more, of a row whose largest result is
0.045 or more.  (2 g^2 + 48) u covers both.
"""
import math

import pytest
import torch

from test_gpu_q8 import B, DT, U, act_64, blank, gen, put, q8, row_scale, untouched  # noqa: F401

pytestmark = pytest.mark.gpu


def rows(g, T, F):
    """Rows between two numbers each, all results of a row small."""
    lo = torch.tensor([-3.0, -5.0, -6.0, -9.0, -12.5, -2.2, -30.0, -0.3], device="cuda")
    hi = torch.tensor([-2.0, -4.0, -5.5, -3.0, -10.0, -0.01, -5.0, 0.3], device="cuda")
    k = torch.arange(T, device="cuda") % len(lo)
    x = torch.rand((T, F), generator=g, device="cuda")
    return lo[k, None] + (hi - lo)[k, None] * x


# every form a row is held in, and the ones that read it again
SIZES = [(8, 1), (16, 9), (8, 300), (9, 513), (8, 2048), (8, 2049), (11, 4103), (8, 8200),
         (8, 16390), (8, 32770), (4099, 700), (4099, 1300)]


@pytest.mark.parametrize("T,F", SIZES)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_results_that_are_all_small(q8, T, F, dt):  # noqa: F811
    g = put(rows(gen(T + F), T, F), DT[dt], 3)
    q, cg, y = blank(T, F, torch.int8), blank(T, F, torch.int8), blank(T, F, torch.float32, 1)
    s, sg = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    q8.cpdp_q8_act("gelu", g, q=q, scale=s, y=y, cg=cg, sg=sg)
    a = act_64("gelu", g.double(), None)
    amax, far = a.abs().amax(1), g.double().square().amax(1)
    slack = (2 * far + 48) * U
    s64 = s.double()
    assert bool((127 * s64 >= amax * (1 - slack)).all())
    assert bool(((127 / 128 * 126.9 * s64 <= amax * (1 + slack)) | (s64 <= 2.0 ** -126)).all())
    off = (q.double() - a / s64[:, None]).abs().amax(1)
    assert bool((off <= 0.5 + 128 * slack).all())
    assert torch.equal(y, q.float() * s[:, None])
    assert torch.equal(sg.double(), row_scale(g))
    untouched(q, cg, y)


def test_rows_beside_ordinary_ones_keep_their_results(q8):  # noqa: F811
    """A row's bits do not depend on the rows beside it."""
    T, F = 64, 500
    g = torch.randn((T, F), generator=gen(1), device="cuda") * 2
    one = []
    for low in (False, True):
        x = g.clone()
        if low:
            x[1::2] = rows(gen(2), T // 2, F)
        q, s = blank(T, F, torch.int8), torch.empty(T, device="cuda")
        q8.cpdp_q8_act("gelu", put(x, torch.float32), q=q, scale=s)
        one.append((q[::2].clone(), s[::2].clone()))
    assert torch.equal(one[0][0], one[1][0]) and torch.equal(one[0][1], one[1][1])
