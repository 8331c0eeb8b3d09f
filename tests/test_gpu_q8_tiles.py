"""Products and gradients of middling sizes, whose tiles of 128 x 128 have a CU to
themselves and are shared by two groups of wavefronts, each with half of every step:
ragged in every direction, at the extremes of 8 bits.

Tolerances: integer sums are exact, their scaling is 3 roundings of u = 2^-24, and bf16
results are the fp32 ones rounded; fp32 sums err by about u sqrt(terms) / 2 of the
result's 2-norm or less (2e-6 covers 16k terms); one rounding to bf16 has a 2-norm of at
most 2^-8 / sqrt(3), and with bf16 results there is one in the sum too.
"""
import math

import pytest
import torch

from test_gpu_q8 import B, DT, U, blank, gen, ints, put, q8, randn, rel, untouched  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K", [(1025, 2100, 1111), (1024, 2048, 1152), (2000, 2000, 2000),
                                   (1153, 2049, 1025), (1000, 4097, 640), (520, 5000, 897),
                                   (2047, 1921, 1409)])
def test_product(q8, M, N, K):  # noqa: F811
    g = gen(M + N + K)
    a, b = put(ints(g, M, K), torch.int8, 20), put(ints(g, N, K), torch.int8, 3)
    sa, sb = torch.rand(M, generator=g, device="cuda"), torch.rand(N, generator=g, device="cuda")
    y = blank(M, N, torch.float32, 5)
    q8.cpdp_q8_matmul(a, sa, b, sb, y)
    want = torch.mm(a.double(), b.double().t().contiguous()) * torch.outer(sa.double(), sb.double())
    assert bool(((y.double() - want).abs() <= 3 * U * want.abs()).all())
    untouched(y)
    # a bf16 result is the fp32 one, rounded once
    half = blank(M, N, torch.bfloat16, 5)
    q8.cpdp_q8_matmul(a, sa, b, sb, half)
    assert torch.equal(half, y.to(torch.bfloat16))
    untouched(half)


@pytest.mark.parametrize("M,N,K", [(500, 4001, 1031), (512, 4096, 1024), (1700, 1100, 2000),
                                   (130, 8190, 1500), (1750, 901, 816)])
def test_product_of_tiles_of_128_x_64(q8, M, N, K):  # noqa: F811
    g = gen(M + 2 * N + K)
    a, b = put(ints(g, M, K), torch.int8, 20), put(ints(g, N, K), torch.int8, 3)
    sa, sb = torch.rand(M, generator=g, device="cuda"), torch.rand(N, generator=g, device="cuda")
    y, half = blank(M, N, torch.float32, 5), blank(M, N, torch.bfloat16, 5)
    q8.cpdp_q8_matmul(a, sa, b, sb, y)
    q8.cpdp_q8_matmul(a, sa, b, sb, half)
    want = torch.mm(a.double(), b.double().t().contiguous()) * torch.outer(sa.double(), sb.double())
    assert bool(((y.double() - want).abs() <= 3 * U * want.abs()).all())
    assert torch.equal(half, y.to(torch.bfloat16))
    untouched(y, half)


def test_product_of_extremes(q8):  # noqa: F811
    M, N, K = 1025, 2100, 1111
    one_m, one_n = torch.ones(M, device="cuda"), torch.ones(N, device="cuda")
    for u, v in ((-128, -128), (127, -128), (127, 127)):
        a = put(torch.full((M, K), u, device="cuda"), torch.int8)
        b = put(torch.full((N, K), v, device="cuda"), torch.int8)
        y = blank(M, N, torch.float32)
        q8.cpdp_q8_matmul(a, one_m, b, one_n, y)
        want = float(torch.tensor(float(u * v * K), dtype=torch.float32))
        assert bool((y == want).all())


@pytest.mark.parametrize("T,N,K", [(1100, 1111, 2100), (1153, 1088, 2049), (2000, 2000, 2000),
                                   (1300, 1281, 1999)])
@pytest.mark.parametrize("dy_dt,out_dt", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"),
                                          ("f32", "bf16")])
def test_grads(q8, T, N, K, dy_dt, out_dt):  # noqa: F811
    g = gen(T + N + K)
    a, b = put(ints(g, T, K), torch.int8, 2), put(ints(g, N, K), torch.int8, 30)
    scales = torch.exp(randn(g, T + N)).to(torch.bfloat16).float()
    sa, sb = scales[:T].contiguous(), scales[T:].contiguous()
    dy = put(randn(g, T, N), DT[dy_dt], 4)
    dx, dw = blank(T, K, DT[out_dt], 6), blank(N, K, DT[out_dt])
    q8.cpdp_q8_grad_input(dy, b, sb, dx)
    q8.cpdp_q8_grad_weight(dy, a, sa, dw)
    want_x = torch.mm(dy.double(), b.double() * sb.double()[:, None])
    want_w = torch.mm(dy.double().t().contiguous(), a.double() * sa.double()[:, None])
    tol = 2e-6 if out_dt == "f32" else math.sqrt(2.0 / 3.0) * B
    assert rel(dx, want_x) <= tol and rel(dw, want_w) <= tol
    untouched(dx, dw)
