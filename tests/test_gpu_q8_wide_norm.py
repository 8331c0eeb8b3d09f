"""The norm's backward pass of a row too wide for one direction of a grid of blocks of 32
columns.  With one row dw is dy h rstd, a product of three numbers (3 roundings of
u = 2^-24, whatever their order), and dx the row's formula (see test_gpu_q8)."""
import pytest
import torch

from test_gpu_q8 import U, gen, q8, randn  # noqa: F401

pytestmark = pytest.mark.gpu


def test_more_than_two_to_the_27_columns(q8):  # noqa: F811
    D = (1 << 27) + 24
    g = gen(8)
    dy, h = randn(g, 1, D), randn(g, 1, D)
    w, rstd = torch.ones(D, device="cuda"), torch.full((1,), 0.75, device="cuda")
    dx, dw = torch.full((1, D), 77.0, device="cuda"), torch.full((D,), 77.0, device="cuda")
    q8.cpdp_q8_norm_bwd(dy, h, w, rstd, dx, dw)
    torch.cuda.synchronize()
    for at in (0, (1 << 26) - 3, D - 5000):
        part = slice(at, at + 5000)
        n = h[0, part].double() * 0.75
        want = dy[0, part].double() * n
        assert bool(((dw[part].double() - want).abs() <= 3 * U * want.abs()).all())
        # the mean of 2^27 products of unit normals is below 2^-9
        assert bool(((dx[0, part].double() - dy[0, part].double() * 0.75).abs()
                     <= n.abs() * 2.0 ** -9 + 1e-6).all())
    assert bool((dw != 77).all()) and bool((dx != 77).all())
