"""Every kernel of the 8-bit path against its operator's definition in 64 bits, at the sizes
of q8_sizes.py (a CPU test sees to it that they take every kernel): random values, ragged
sizes, padding that a stray read or write would show, results that repeat bit by bit.

Tolerances, with u = 2^-24 and b = 2^-8, as test_gpu_q8 derives them; where it has none:
* dw of the norm's backward pass: two roundings a term; the rows of a group one after the
  other, T / 1024 of them at most, rounded up; 3 additions of a block's wavefronts; 1024
  parts by 32 threads a column, 32 additions each, and 5 across the threads.
* An element of a gradient: R u of its terms' sizes for R fp32 additions in any order, 2 u
  for the scaling, b for terms that are rounded to one bfloat16 number (cpdp_q8.h says
  where), and a bf16 result's own rounding.
"""
import math

import pytest
import torch

import q8_sizes
from q8_sizes import BF16, TYPES
from test_gpu_q8 import (B, U, act_64, act_bwd_64, blank, check_held, gen, ints,  # noqa: F401
                         norm_bwd_64, put, q8, randn, rel, row_scale, untouched)

pytestmark = pytest.mark.gpu

DTYPE = (torch.float32, torch.bfloat16)


def name(case):
    return "-".join(map(str, case))


def vec(n):
    return torch.full((n,), 77.0, device="cuda")


def near_halves(q, v, s, slack):
    """|q - v / s| <= 1/2 and the quotient's roundings, v known to `slack`."""
    off = (q.double() - v / s.double()[:, None]).abs()
    assert float(off.max()) <= 0.5 + 128 * slack


@pytest.mark.parametrize("T,D", q8_sizes.ROWS)
@pytest.mark.parametrize("x_dt,y_dt", TYPES)
def test_rows_and_values(q8, T, D, x_dt, y_dt):  # noqa: F811
    g = gen(T + D)
    x = put(randn(g, T, D) * torch.exp(3 * randn(g, T, 1)), DTYPE[x_dt], 3)
    q, y, s = blank(T, D, torch.int8, 5), blank(T, D, DTYPE[y_dt], 1), vec(T)
    q8.cpdp_q8_rows(x, q, s, y=y)
    want = row_scale(x)
    assert torch.equal(s.double(), want)
    quotient = x.double() / want[:, None]
    if x_dt == BF16:
        assert torch.equal(q.double(), torch.round(quotient))
    near_halves(q, x.double(), s, U)
    held = q.float() * s[:, None]
    assert torch.equal(y, held.to(DTYPE[y_dt]))
    back = blank(T, D, DTYPE[y_dt], 2)
    q8.cpdp_q8_values(q, s, back)
    assert torch.equal(back, y)
    untouched(q, y, back)


@pytest.mark.parametrize("T,D", q8_sizes.ROWS)
@pytest.mark.parametrize("dt,w_dt", TYPES)
@pytest.mark.parametrize("res", [True, False])
def test_norm(q8, T, D, dt, w_dt, res):  # noqa: F811
    g, eps = gen(T + D + 1), 1e-5
    x = put(randn(g, T, D) * torch.exp(randn(g, T, 1)), DTYPE[dt], 8)
    r = put(randn(g, T, D), DTYPE[dt]) if res else None
    w = (1 + 0.2 * randn(g, D)).to(DTYPE[w_dt])
    h = blank(T, D, DTYPE[dt], 4) if res else None
    q, y, s, rstd = blank(T, D, torch.int8), blank(T, D, DTYPE[w_dt]), vec(T), vec(T)
    q8.cpdp_q8_norm(x, w, eps, q=q, scale=s, residual=r, h=h, rstd=rstd, y=y)
    if res:
        assert torch.equal(h, (x.float() + r.float()).to(DTYPE[dt]))
        untouched(h)
    hh = (h if res else x).double()
    want = (hh.square().mean(1) + eps).rsqrt()
    assert float((rstd.double() / want - 1).abs().max()) <= 32 * U
    check_held(q, s, hh * w.double() * want[:, None], 40 * U)
    assert torch.equal(y, (q.float() * s[:, None]).to(DTYPE[w_dt]))
    untouched(q, y)


@pytest.mark.parametrize("T,D", q8_sizes.NORM_BWD)
@pytest.mark.parametrize("dt,w_dt", TYPES)
@pytest.mark.parametrize("res", [True, False])
def test_norm_bwd(q8, T, D, dt, w_dt, res):  # noqa: F811
    g = gen(T + D)
    dy, h = put(randn(g, T, D), DTYPE[dt], 2), put(2 * randn(g, T, D), DTYPE[dt], 9)
    dres = put(randn(g, T, D), DTYPE[dt]) if res else None
    w = (1 + 0.2 * randn(g, D)).to(DTYPE[w_dt])
    rstd = (h.double().square().mean(1) + 1e-6).rsqrt().float()
    out = []
    for _ in range(2):
        dx, dw = blank(T, D, DTYPE[dt], 3), vec(D).to(DTYPE[w_dt])
        q8.cpdp_q8_norm_bwd(dy, h, w, rstd, dx, dw, dres=dres)
        out.append((dx, dw))
    want, size, want_w, size_w = norm_bwd_64(dy, h, w, rstd, dres)
    over = B * want.abs() if dt == BF16 else 0
    assert bool(((dx.double() - want).abs() <= 72 * U * size + over + 1e-37).all())
    over = B * want_w.abs() if w_dt == BF16 else 0
    steps = 2 + math.ceil(T / 1024) + 3 + 32 + 5
    # (a bf16 result rounds what the sum left, not the exact one)
    slack = steps * U * size_w * 1.01
    assert bool(((dw.double() - want_w).abs() <= slack + over + 1e-37).all())
    untouched(dx)
    assert torch.equal(out[0][0], dx) and torch.equal(out[0][1], dw)


@pytest.mark.parametrize("T,F", q8_sizes.ROWS)
@pytest.mark.parametrize("kind", ["gelu", "swiglu"])
@pytest.mark.parametrize("dt,y_dt", TYPES)
def test_activations(q8, T, F, kind, dt, y_dt):  # noqa: F811
    gen_ = gen(T + F)
    gated = kind == "swiglu"
    g = put(3 * randn(gen_, T, F), DTYPE[dt], 5)
    u = put(randn(gen_, T, F), DTYPE[dt], 5) if gated else None
    q, cg = blank(T, F, torch.int8), blank(T, F, torch.int8, 3)
    cu = blank(T, F, torch.int8, 3) if gated else None
    y, s, sg, su = blank(T, F, DTYPE[y_dt]), vec(T), vec(T), vec(T) if gated else None
    q8.cpdp_q8_act(kind, g, u, q=q, scale=s, y=y, cg=cg, sg=sg, cu=cu, su=su)
    a = act_64(kind, g.double(), u.double() if gated else None)
    slack = 32 * U
    assert bool((127 * s.double() >= a.abs().amax(1) * (1 - slack)).all())
    near_halves(q, a, s, slack)
    assert torch.equal(y, (q.float() * s[:, None]).to(DTYPE[y_dt]))
    for x, c, sc in ((g, cg, sg), (u, cu, su)):
        if x is not None:
            assert torch.equal(sc.double(), row_scale(x))
            near_halves(c, x.double(), sc, U)
            untouched(c)
    untouched(q, y)
    da = put(randn(gen_, T, F), DTYPE[dt])
    dg, du = blank(T, F, DTYPE[dt], 1), blank(T, F, DTYPE[dt], 1) if gated else None
    q8.cpdp_q8_act_bwd(kind, da, cg, sg, dg, cu=cu, su=su, du=du)
    G = cg.double() * sg.double()[:, None]
    Uv = cu.double() * su.double()[:, None] if gated else None
    want_g, want_u = act_bwd_64(kind, da.double(), G, Uv)
    results = [(dg, want_g, da.double().abs() * (Uv.abs() if gated else 1.0) * (1 + G.abs()))]
    if gated:
        results.append((du, want_u, da.double().abs() * G.abs() * (1 + G.abs())))
    for got, want, size in results:
        over = B * want.abs() if dt == BF16 else 0
        assert bool(((got.double() - want).abs() <= 32 * U * size + over + 1e-37).all())
        untouched(got)


@pytest.mark.parametrize("M,N,K", q8_sizes.PRODUCTS)
def test_product(q8, M, N, K):  # noqa: F811
    g = gen(M + N + K)
    a, b = put(ints(g, M, K), torch.int8, 7), put(ints(g, N, K), torch.int8)
    sa, sb = torch.rand(M, generator=g, device="cuda"), torch.rand(N, generator=g, device="cuda")
    y, half = blank(M, N, torch.float32, 3), blank(M, N, torch.bfloat16, 3)
    q8.cpdp_q8_matmul(a, sa, b, sb, y)
    q8.cpdp_q8_matmul(a, sa, b, sb, half)
    want = torch.mm(a.double(), b.double().t().contiguous()) * sa.double()[:, None] * sb.double()
    assert bool(((y.double() - want).abs() <= 3 * U * want.abs() + 1e-30).all())
    assert torch.equal(half, y.to(torch.bfloat16))
    untouched(y, half)


@pytest.mark.parametrize("case", q8_sizes.GRADS, ids=name)
def test_gradients(q8, case):  # noqa: F811
    op, T, N, K, dy_dt, out_dt = case
    g = gen(T + N + K)
    R, C = (N, T) if op == "grad_input" else (T, N)  # what is summed, rows of the result
    held = put(ints(g, R, K), torch.int8, 18)
    scale = torch.exp(randn(g, R)).to(torch.bfloat16).float()
    dy = put(randn(g, T, N), DTYPE[dy_dt], 4)
    call = q8.cpdp_q8_grad_input if op == "grad_input" else q8.cpdp_q8_grad_weight
    out, again = blank(C, K, DTYPE[out_dt], 6), blank(C, K, DTYPE[out_dt], 6)
    call(dy, held, scale, out)
    call(dy, held, scale, again)
    left = dy.double() if op == "grad_input" else dy.double().t().contiguous()
    right = held.double() * scale.double()[:, None]
    want, size = torch.mm(left, right), torch.mm(left.abs(), right.abs())
    assert rel(out, want) <= (2e-6 if out_dt != BF16 else math.sqrt(2.0 / 3.0) * B)
    slack = ((B if out_dt == BF16 and R > 64 else 0.0) + (R + 2) * U) * size
    if out_dt == BF16:
        slack = slack + B * (want.abs() + slack)
    assert bool(((out.double() - want).abs() <= slack).all())
    untouched(out)
    assert torch.equal(out, again)
