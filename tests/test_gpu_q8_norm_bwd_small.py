"""The norm's backward pass on both sides of the line between one launch and two: the
same results by float64's measure, rows and columns at the edges of its blocks, a scale
that is not finite, and results that do not change from call to call.

Tolerances as in test_gpu_q8: a row's sum takes at most 64 roundings of u = 2^-24, dw's
at most 8 a thread and 20 across threads, beside those of its terms; bf16 results one
rounding more, of up to 2^-8 of the value.
"""
import math

import pytest
import torch

from test_gpu_q8 import B, DT, U, blank, gen, put, q8, randn, untouched  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,D", [(1, 8), (255, 9), (256, 512), (257, 513), (1023, 384), (1025, 384),
                                 (2048, 200), (2049, 200), (64, 4096), (64, 4097), (96, 4088),
                                 (100, 4096), (2047, 380), (1576, 384)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("w_dt,dres", [("f32", True), ("bf16", False)])
def test_against_float64(q8, T, D, dt, w_dt, dres):  # noqa: F811
    g = gen(T + 3 * D)
    dy, h = put(randn(g, T, D), DT[dt], 5), put(randn(g, T, D), DT[dt], 9)
    r = put(randn(g, T, D), DT[dt]) if dres else None
    w = randn(g, D).to(DT[w_dt])
    rstd = torch.rand(T, generator=g, device="cuda") + 0.5
    dx, dw = blank(T, D, DT[dt], 3), torch.empty(D, dtype=DT[w_dt], device="cuda")
    q8.cpdp_q8_norm_bwd(dy, h, w, rstd, dx, dw, dres=r)
    untouched(dx)
    n = h.double() * rstd.double()[:, None]
    dn = dy.double() * w.double()
    mean = (dn * n).mean(1, keepdim=True)
    want = (dn - n * mean) * rstd.double()[:, None]
    if dres:
        want = want + r.double()
    # the mean's error, and those of the products and sums it goes into
    size = (dn * n).abs().mean(1, keepdim=True)
    slack = (n.abs() * (64 * U * size + 4 * U * mean.abs()) + 6 * U * dn.abs()) * \
        rstd.double()[:, None] + 2 * U * want.abs() + (2 * U * r.double().abs() if dres else 0)
    if dt == "bf16":
        slack = slack + B * (want.abs() + slack)
    assert bool(((dx.double() - want).abs() <= slack).all())
    want = (dy.double() * n).sum(0)
    slack = 32 * U * (dy.double() * n).abs().sum(0) + (B * want.abs() if w_dt == "bf16" else 0)
    assert bool(((dw.double() - want).abs() <= slack * 1.01).all())
    dx2, dw2 = blank(T, D, DT[dt], 3), torch.empty_like(dw)
    q8.cpdp_q8_norm_bwd(dy, h, w, rstd, dx2, dw2, dres=r)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)


def test_a_row_that_is_not_finite(q8):  # noqa: F811
    T, D = 300, 130
    g = gen(3)
    dy, h = put(randn(g, T, D), torch.float32), put(randn(g, T, D), torch.float32)
    h[7, 5] = math.inf
    w, rstd = randn(g, D), torch.ones(T, device="cuda")
    dx, dw = blank(T, D, torch.float32), torch.empty(D, device="cuda")
    q8.cpdp_q8_norm_bwd(dy, h, w, rstd, dx, dw)
    rows = torch.arange(T, device="cuda") != 7
    cols = torch.arange(D, device="cuda") != 5
    assert bool(torch.isfinite(dx[rows]).all()) and not bool(torch.isfinite(dx[7]).any())
    assert bool(torch.isfinite(dw[cols]).all()) and not math.isfinite(float(dw[5]))
