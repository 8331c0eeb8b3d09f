"""How many bits of what they sum the gradients of a product keep, as cpdp_q8.h says it: all
of them with scales of 8 significant bits, within 2^-16 with bf16 dy and any other scales,
within 2^-8 with bf16 results of long sums.

A bound beside each: R 2^-24 of the sum of the terms' sizes for R fp32 additions in any
order, 2 u for the scaled value's rounding, and a bf16 result's own rounding.
"""
import pytest
import torch

from test_gpu_q8 import B, DT, U, blank, gen, ints, put, q8, randn, untouched  # noqa: F401

pytestmark = pytest.mark.gpu

# few tokens, the operands as they lie, laid out, and several tiles
SIZES = [(3, 70, 100), (20, 300, 130), (60, 100, 64), (200, 130, 70), (1100, 300, 260)]


@pytest.mark.parametrize("T,N,K", SIZES)
@pytest.mark.parametrize("dy_dt,out_dt", [("bf16", "f32"), ("f32", "f32"), ("bf16", "bf16"),
                                          ("f32", "bf16")])
@pytest.mark.parametrize("eight_bits", [True, False])
def test_bits_that_are_kept(q8, T, N, K, dy_dt, out_dt, eight_bits):  # noqa: F811
    g = gen(T + N + K)
    a, b = put(ints(g, T, K), torch.int8, 2), put(ints(g, N, K), torch.int8, 30)
    scales = torch.exp(randn(g, T + N))
    if eight_bits:
        scales = scales.to(torch.bfloat16).float()
    sa, sb = scales[:T].contiguous(), scales[T:].contiguous()
    dy = put(randn(g, T, N), DT[dy_dt], 4)
    dx, dw = blank(T, K, DT[out_dt], 6), blank(N, K, DT[out_dt])
    q8.cpdp_q8_grad_input(dy, b, sb, dx)
    q8.cpdp_q8_grad_weight(dy, a, sa, dw)
    untouched(dx, dw)
    for got, left, right, R in ((dx, dy.double(), b.double() * sb.double()[:, None], N),
                                (dw, dy.double().t().contiguous(),
                                 a.double() * sa.double()[:, None], T)):
        want, size = torch.mm(left, right), torch.mm(left.abs(), right.abs())
        if out_dt == "bf16" and R > 64:
            kept = B
        elif dy_dt == "bf16" and not eight_bits:
            kept = 2.0 ** -16
        else:
            kept = 0.0
        slack = (kept + (R + 2) * U) * size
        if out_dt == "bf16":
            slack = slack + B * (want.abs() + slack)
        assert bool(((got.double() - want).abs() <= slack).all())


def test_a_long_sum_that_cancels_is_there_in_fp32(q8):  # noqa: F811
    """The choice that the header names: an fp32 result of a sum whose terms cancel."""
    T, N, K = 200, 512, 96
    g = gen(3)
    b = put(ints(g, N // 2, K).repeat_interleave(2, 0), torch.int8)
    sb = torch.exp(randn(g, N // 2)).to(torch.bfloat16).float().repeat_interleave(2)
    dy = randn(g, T, N // 2).to(torch.bfloat16).float().repeat_interleave(2, 1)
    dy[:, 1::2] *= -1
    dy[:, 0] += 0.5
    dy = put(dy, torch.bfloat16)
    dx = blank(T, K, torch.float32)
    q8.cpdp_q8_grad_input(dy, b, sb, dx)
    want = torch.mm(dy.double(), b.double() * sb.double()[:, None])
    size = torch.mm(dy.double().abs(), b.double().abs() * sb.double()[:, None])
    assert bool(((dx.double() - want).abs() <= (N + 2) * U * size).all())
