"""fp32 gradients of a product at sizes where dy is read as it is and taken apart on
its way to the matrix cores, rather than laid out first: ragged sizes, sums cut into
slices, values at fp32's ends, and padding that holds NaN.

Tolerance: the scaled gradient's three parts are exact, so the error is that of fp32
sums, whose 2-norm over the result's is about u sqrt(terms) / 2 or less: 2e-6 covers 16k
terms (u = 2^-24).
"""
import math

import pytest
import torch

from test_gpu_q8 import U, blank, gen, ints, put, q8, randn, rel, untouched  # noqa: F401

pytestmark = pytest.mark.gpu

# T, N, K; both gradients sum over about a thousand values where K is small
SIZES = [(1001, 1003, 71), (1576, 1536, 384), (640, 1250, 64), (1250, 641, 65), (960, 2047, 1),
         (4000, 600, 100), (400, 1536, 384), (1576, 1153, 385)]


def both(q8, dy, a, sa, b, sb, out_dt=torch.float32):  # noqa: F811
    T, N = dy.shape
    K = a.shape[1]
    dx, dw = blank(T, K, out_dt, 6), blank(N, K, out_dt)
    q8.cpdp_q8_grad_input(dy, b, sb, dx)
    q8.cpdp_q8_grad_weight(dy, a, sa, dw)
    untouched(dx, dw)
    return dx, dw


@pytest.mark.parametrize("T,N,K", SIZES)
def test_sizes(q8, T, N, K):  # noqa: F811
    g = gen(T + 2 * N + 3 * K)
    a, b = put(ints(g, T, K), torch.int8, 2), put(ints(g, N, K), torch.int8, 30)
    sa, sb = torch.rand(T, generator=g, device="cuda"), torch.rand(N, generator=g, device="cuda")
    dy = put(randn(g, T, N), torch.float32, 4)
    dy._base[:, N:] = math.nan
    dx, dw = both(q8, dy, a, sa, b, sb)
    want_x = torch.mm(dy.double(), b.double() * sb.double()[:, None])
    want_w = torch.mm(dy.double().t().contiguous(), a.double() * sa.double()[:, None])
    assert rel(dx, want_x) <= 2e-6 and rel(dw, want_w) <= 2e-6
    # the same bits again
    dx2, dw2 = both(q8, dy, a, sa, b, sb)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)


@pytest.mark.parametrize("at", [0, 517, 1000])
def test_values_at_the_ends(q8, at):  # noqa: F811
    """An infinity, a NaN and numbers past bfloat16's largest one reach what depends on
    them and nothing else, wherever in the sum they stand."""
    T, N, K = 1001, 1003, 71
    g = gen(at)
    a, b = put(ints(g, T, K), torch.int8), put(ints(g, N, K), torch.int8)
    a[:, 0], b[:, 0] = 1, 1
    one_t, one_n = torch.ones(T, device="cuda"), torch.ones(N, device="cuda")
    dy = randn(g, T, N)
    dy[2, at], dy[4, at] = math.inf, math.nan
    dx, _ = both(q8, put(dy, torch.float32), a, one_t, b, one_n)
    rows = torch.arange(T, device="cuda")
    assert bool(torch.isfinite(dx[(rows != 2) & (rows != 4)]).all())
    assert float(dx[2, 0]) == math.inf and bool(torch.isnan(dx[4]).all())

    dy = randn(g, T, N)
    dy[at, 3], dy[at, 5] = -math.inf, math.nan
    _, dw = both(q8, put(dy, torch.float32), a, one_t, b, one_n)
    chans = torch.arange(N, device="cuda")
    assert bool(torch.isfinite(dw[(chans != 3) & (chans != 5)]).all())
    assert float(dw[3, 0]) == -math.inf and bool(torch.isnan(dw[5]).all())

    dy = torch.zeros(T, N, device="cuda")
    dy[1, at], dy[at, 1] = 3.4e38, -3.4e38  # both round past the largest bfloat16
    if at == 1:
        dy[1, 1] = 3.4e38
    dx, dw = both(q8, put(dy, torch.float32), a, one_t, b, one_n)
    assert abs(float(dx[1, 0]) / 3.4e38 - 1) <= 4 * U
    assert abs(float(dw[1, 0]) / -3.4e38 - 1) <= 4 * U


def test_each_term_to_fp32(q8):  # noqa: F811
    """A sum of one value that is not zero is that value's product, of which nothing is
    lost but the scale's and the sum's roundings."""
    T, N, K = 1001, 1003, 71
    g = gen(5)
    a, b = put(ints(g, T, K), torch.int8), put(ints(g, N, K), torch.int8)
    sa = torch.rand(T, generator=g, device="cuda") + 0.5
    sb = torch.rand(N, generator=g, device="cuda") + 0.5
    dy = torch.zeros(T, N, device="cuda")
    place = torch.arange(T, device="cuda")
    vals = randn(g, T)
    dy[place, place] = vals  # one a row and, of the first T columns, one a column
    dx, dw = both(q8, put(dy, torch.float32), a, sa, b, sb)
    want = vals.double()[:, None] * sb.double()[:T, None] * b.double()[:T]
    assert bool(((dx.double() - want).abs() <= 4 * U * want.abs()).all())
    want = vals.double()[:, None] * sa.double()[:, None] * a.double()
    assert bool(((dw.double()[:T] - want).abs() <= 4 * U * want.abs()).all())
    assert bool((dw[T:] == 0).all())
