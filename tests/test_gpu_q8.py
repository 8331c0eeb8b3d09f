"""The 8-bit activation path against its definitions in 64 bits: row shapes on
both sides of every switch, ragged rows, slices of wider matrices, rows that are
zero or not finite, empty inputs, streams, captured graphs, offsets past 32
bits, and gradients against differences.

Tolerances.  u = 2^-24 is fp32's unit roundoff and b = 2^-8 bfloat16's.
* Whole numbers: q is x / s, rounded: |q - x / s| <= 1/2 plus the roundings of
  x / s itself; bf16 inputs of a row quantiser have none.
* A norm's sum takes at most 64 roundings (32 terms a thread, 6 steps across a
  wavefront, 16 wavefronts, the division and the root, which halves them).
* A product of 8-bit numbers is exact; converting and scaling it are 3 roundings.
* Sums on the matrix cores: the error's 2-norm over the result's, with random
  signs, is about u sqrt(terms) / 2 or less; 2e-6 covers 16k terms.
* One rounding to bfloat16 has a 2-norm of at most b / sqrt(3).
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U, B = 2.0 ** -24, 2.0 ** -8
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SMALLEST = 2.0 ** -126


@pytest.fixture(scope="module")
def q8():
    from paper_2607_21224_amd import q8 as m
    return m


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def put(x, dtype, pad=0):
    """x as rows with aligned starts, `pad` further elements a row, all padding
    set to a value that a stray read would show."""
    T, D = x.shape
    size = torch.empty((), dtype=dtype).element_size()
    ld = (D + pad + 16 // size - 1) // (16 // size) * (16 // size)
    full = torch.full((T, ld), 77.0 if dtype != torch.int8 else 77, device="cuda").to(dtype)
    full[:, :D] = x.to(dtype)
    return full[:, :D]


def blank(T, D, dtype, pad=0):
    return put(torch.zeros((T, D), device="cuda"), dtype, pad)


def padding(v):
    """What lies between the rows of a tensor that put() made."""
    return v._base[:, v.shape[1]:]


def untouched(*vs):
    for v in vs:
        assert bool((padding(v).float() == 77).all())


def row_scale(v):
    """The definition, on the CPU in 64 bits."""
    out = []
    for a in v.double().abs().amax(1).tolist():
        if not math.isfinite(a):
            out.append(math.nan)
            continue
        m, e = math.frexp(a / 127.0) if a > 0 else (0.0, 0)
        s = math.ldexp(math.ceil(m * 256.0), e - 8)
        # the quotient is rounded: step down where a smaller scale still does
        m2, e2 = math.frexp(s) if s > 0 else (0.0, 0)
        down = s - math.ldexp(1.0, e2 - 8)
        if s > 0 and 127.0 * down >= a:
            s = down
        out.append(max(s, SMALLEST))
    return torch.tensor(out, dtype=torch.float64, device=v.device)


def check_held(q, s, v, slack):
    """8-bit rows against v (64 bits), each v known to a relative `slack`."""
    a = v.abs().amax(1)
    s64 = s.double()
    bits = s.view(torch.int32)
    assert bool((bits & 0xFFFF == 0).all())  # 8 significant bits
    assert bool((127 * s64 >= a * (1 - slack)).all())
    below = (bits - 0x10000).view(torch.float32).double()
    assert bool(((127 * below < a * (1 + slack)) | (s64 <= SMALLEST)).all())
    off = (q.double() - v / s64[:, None]).abs()
    assert float(off.max()) <= 0.5 + 128 * (slack + U)
    assert int(q.abs().max()) <= 127


def rel(x, y):
    n = float(y.double().norm())
    d = float((x.double() - y.double()).norm())
    return d / n if n else d


# both sides of every switch of the row shapes
WIDTHS = [1, 7, 8, 9, 511, 512, 513, 1024, 1025, 2047, 2049, 4096, 4103, 8192, 8195, 16385, 32769]


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_rows_and_values(q8, D, dt):
    T = 5
    x = put(randn(gen(D), T, D) * torch.tensor([1e-3, 1.0, 50.0, 0.0, 1e4],
                                               device="cuda")[:, None], DT[dt], pad=3)
    q, y = blank(T, D, torch.int8, 5), blank(T, D, torch.bfloat16, 1)
    s = torch.empty(T, device="cuda")
    q8.cpdp_q8_rows(x, q, s, y=y)
    want = row_scale(x)
    assert torch.equal(s.double(), want)
    quotient = x.double() / want[:, None]
    if dt == "bf16":
        assert torch.equal(q.double(), torch.round(quotient))
    assert float((q.double() - quotient).abs().max()) <= 0.5 + 127 * U
    held = q.float() * s[:, None]
    assert torch.equal(y, held.to(torch.bfloat16))
    back = blank(T, D, torch.float32, 2)
    q8.cpdp_q8_values(q, s, back)
    assert torch.equal(back, held)
    untouched(q, y, back)


@pytest.mark.parametrize("D", [300, 700, 1300, 2048])
def test_rows_of_many_tokens(q8, D):
    """From 1024 rows on a wavefront holds a row of up to 2048 elements."""
    T = 1027
    x = put(randn(gen(D), T, D), torch.bfloat16)
    q, s = blank(T, D, torch.int8), torch.empty(T, device="cuda")
    q8.cpdp_q8_rows(x, q, s)
    want = row_scale(x)
    assert torch.equal(s.double(), want)
    assert torch.equal(q.double(), torch.round(x.double() / want[:, None]))


def test_scale_at_exact_quotients(q8):
    """Rows whose largest element is 127 times a bfloat16 number, or the fp32
    number after or before it, and ties between two whole numbers."""
    tops = []
    for e in (-120, -3, 0, 9, 100):
        for m in (128, 129, 200, 255):
            t = torch.tensor(127.0 * m * 2.0 ** (e - 7))
            tops += [t, torch.nextafter(t, torch.tensor(math.inf)),
                     torch.nextafter(t, torch.tensor(0.0))]
    top = torch.stack(tops).cuda()
    k = torch.arange(1, 127, device="cuda") + 0.5
    x = torch.cat([top[:, None], (top / 127)[:, None] * k], 1)
    q, s = blank(*x.shape, torch.int8), torch.empty(len(top), device="cuda")
    x = put(x, torch.float32)
    q8.cpdp_q8_rows(x, q, s)
    want = row_scale(x)
    assert torch.equal(s.double(), want)
    exact = (x.double() / want[:, None])
    assert torch.equal(q.double(), torch.round(exact.float().double()))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_rows_that_are_not_finite(q8, dt):
    D = 600
    x = randn(gen(1), 6, D)
    x[0, 5] = math.inf
    x[1, 599] = -math.inf
    x[2, 0] = math.nan
    x[3] = 0
    x[4] = 1e-42  # below the smallest scale's half step
    x = put(x, DT[dt])
    q, s = blank(6, D, torch.int8), torch.empty(6, device="cuda")
    y = blank(6, D, torch.float32)
    q8.cpdp_q8_rows(x, q, s, y=y)
    assert bool(torch.isnan(s[:3]).all()) and bool((q[:3] == 0).all())
    assert bool(torch.isnan(y[:3]).all())
    assert float(s[3]) == SMALLEST == float(s[4]) and bool((q[3:5] == 0).all())
    assert bool(torch.isfinite(y[5]).all())


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("dt,w_dt,res", [("f32", "f32", True), ("bf16", "f32", True),
                                         ("bf16", "bf16", False), ("f32", "bf16", False)])
def test_norm(q8, D, dt, w_dt, res):
    T, g, eps = 3, gen(D + 1), 1e-5
    x = put(randn(g, T, D) * 3, DT[dt], 8)
    r = put(randn(g, T, D), DT[dt]) if res else None
    w = (1 + 0.2 * randn(g, D)).to(DT[w_dt])
    h = blank(T, D, DT[dt], 4) if res else None
    q, y = blank(T, D, torch.int8), blank(T, D, torch.bfloat16)
    s, rstd = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    q8.cpdp_q8_norm(x, w, eps, q=q, scale=s, residual=r, h=h, rstd=rstd, y=y)
    if res:
        assert torch.equal(h, (x.float() + r.float()).to(DT[dt]))
        untouched(h)
    hh = (h if res else x).double()
    want = (hh.square().mean(1) + eps).rsqrt()
    assert float((rstd.double() / want - 1).abs().max()) <= 32 * U
    check_held(q, s, hh * w.double() * want[:, None], 40 * U)
    assert torch.equal(y, (q.float() * s[:, None]).to(torch.bfloat16))
    untouched(q, y)


def test_norm_in_place_and_without_extras(q8):
    T, D = 70, 384
    x, r = put(randn(gen(2), T, D), torch.bfloat16), put(randn(gen(3), T, D), torch.bfloat16)
    w = torch.ones(D, device="cuda")
    out = []
    for h in (blank(T, D, torch.bfloat16), r.clone(), x.clone()):
        xx, rr = x.clone(), r.clone()
        # h apart, then the residual's own rows, then the input's own rows
        target = h if not out else (rr if len(out) == 1 else xx)
        q, s = blank(T, D, torch.int8), torch.empty(T, device="cuda")
        q8.cpdp_q8_norm(xx, w, 0.0, q=q, scale=s, residual=rr, h=target)
        out.append((target.clone(), q.clone(), s.clone()))
    for other in out[1:]:
        for a, b in zip(out[0], other):
            assert torch.equal(a, b)


def test_norm_rows_that_are_not_finite(q8):
    D = 1000
    x = randn(gen(4), 4, D)
    x[0, 3], x[1, 999], x[2] = math.inf, math.nan, 0
    x = put(x, torch.float32)
    q, s = blank(4, D, torch.int8), torch.empty(4, device="cuda")
    y = blank(4, D, torch.bfloat16)
    q8.cpdp_q8_norm(x, torch.ones(D, device="cuda"), 1e-6, q=q, scale=s, y=y)
    assert bool(torch.isnan(y[:2]).all()) and bool((q[:3] == 0).all())
    assert bool((y[2] == 0).all()) and bool(torch.isfinite(y[3]).all())
    # a weight that is not finite reaches every row
    w = torch.ones(D, device="cuda")
    w[7] = math.nan
    q8.cpdp_q8_norm(x, w, 1e-6, q=q, scale=s, y=y)
    assert bool(torch.isnan(s).all())


def norm_bwd_64(dy, h, w, rstd, dres):
    n = h.double() * rstd.double()[:, None]
    g = dy.double() * w.double()
    c = (g * n).mean(1, keepdim=True)
    dx = (g - n * c) * rstd.double()[:, None]
    size = (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True)) * rstd.double()[:, None]
    if dres is not None:
        dx = dx + dres.double()
        size = size + dres.double().abs()
    return dx, size, (dy.double() * n).sum(0), (dy.double() * n).abs().sum(0)


@pytest.mark.parametrize("T,D", [(1, 1), (3, 7), (70, 384), (1576, 387), (37, 513), (20, 2049),
                                 (11, 4100), (9, 8200), (5, 16390), (2100, 64)])
@pytest.mark.parametrize("dt,w_dt,res", [("f32", "f32", True), ("bf16", "bf16", False),
                                         ("bf16", "f32", True)])
def test_norm_bwd(q8, T, D, dt, w_dt, res):
    g = gen(T + D)
    dy, h = put(randn(g, T, D), DT[dt], 2), put(2 * randn(g, T, D), DT[dt], 9)
    dres = put(randn(g, T, D), DT[dt]) if res else None
    w = (1 + 0.2 * randn(g, D)).to(DT[w_dt])
    rstd = (h.double().square().mean(1) + 1e-6).rsqrt().float()
    dx, dw = blank(T, D, DT[dt], 3), torch.empty(D, dtype=DT[w_dt], device="cuda")
    q8.cpdp_q8_norm_bwd(dy, h, w, rstd, dx, dw, dres=dres)
    want, size, want_w, size_w = norm_bwd_64(dy, h, w, rstd, dres)
    over = B * want.abs() if dt == "bf16" else 0
    assert bool(((dx.double() - want).abs() <= 72 * U * size + over + 1e-37).all())
    # rows of a part, parts of a thread, threads of a column
    over = B * want_w.abs() if w_dt == "bf16" else 0
    steps = 8 + T / 1024 + 1024 * 4 / 16 + 16
    assert bool(((dw.double() - want_w).abs() <= steps * U * size_w + over + 1e-37).all())
    untouched(dx)


def test_norm_bwd_against_differences(q8):
    """The norm's derivative along a direction, by central differences of the
    norm in 64 bits (before the rounding to 8 bits, which passes gradients on)."""
    T, D, eps, step = 17, 400, 1e-5, 1e-5
    g = gen(9)
    h, dy = put(randn(g, T, D), torch.float32), put(randn(g, T, D), torch.float32)
    w = 1 + 0.3 * randn(g, D)
    q, s, rstd = blank(T, D, torch.int8), torch.empty(T, device="cuda"), torch.empty(
        T, device="cuda")
    q8.cpdp_q8_norm(h, w, eps, q=q, scale=s, rstd=rstd)
    dx, dw = blank(T, D, torch.float32), torch.empty(D, device="cuda")
    q8.cpdp_q8_norm_bwd(dy, h, w, rstd, dx, dw)

    def loss(hh, ww):
        return float((hh * (hh.square().mean(1, keepdim=True) + eps).rsqrt() * ww *
                      dy.double()).sum())

    for k in range(4):
        d, dwd = randn(g, T, D).double(), randn(g, D).double()
        h64, w64 = h.double(), w.double()
        by_h = (loss(h64 + step * d, w64) - loss(h64 - step * d, w64)) / (2 * step)
        by_w = (loss(h64, w64 + step * dwd) - loss(h64, w64 - step * dwd)) / (2 * step)
        # the differences' own error is step^2 and 2^-52 / step of the loss' terms
        scale = float(dx.double().norm() * d.norm()) + float(dw.double().norm() * dwd.norm())
        assert abs(float((dx.double() * d).sum()) - by_h) <= 1e-6 * scale
        assert abs(float((dw.double() * dwd).sum()) - by_w) <= 1e-6 * scale


def ints(g, *shape):
    return torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=torch.int8)


PRODUCTS = [(1, 1, 1), (1, 4096, 4096), (2, 100, 33), (5, 17, 500), (16, 1000, 129),
            (17, 96, 1024), (33, 70, 4096), (64, 256, 128), (65, 63, 127), (100, 515, 385),
            (197, 1536, 384), (600, 130, 2000), (1576, 1153, 385), (1, 50, 131071),
            (1800, 2000, 640), (4096, 4100, 200)]


@pytest.mark.parametrize("M,N,K", PRODUCTS)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_product(q8, M, N, K, dt):
    g = gen(M + N + K)
    a, b = put(ints(g, M, K), torch.int8, 7), put(ints(g, N, K), torch.int8)
    sa, sb = torch.rand(M, generator=g, device="cuda"), torch.rand(N, generator=g, device="cuda")
    y = blank(M, N, DT[dt], 3)
    q8.cpdp_q8_matmul(a, sa, b, sb, y)
    want = torch.mm(a.double(), b.double().t().contiguous()) * sa.double()[:, None] * sb.double()
    tol = 4 * U + (B if dt == "bf16" else 0)
    assert bool(((y.double() - want).abs() <= tol * want.abs() + 1e-30).all())
    untouched(y)


@pytest.mark.parametrize("M", [1, 40, 300])
def test_product_of_extremes(q8, M):
    """The largest sums there are: -128 times -128, 131071 times."""
    K, N = 131071, 20
    a, b = (torch.full((r, K), -128, dtype=torch.int8, device="cuda") for r in (M, N))
    a, b = put(a, torch.int8), put(b, torch.int8)
    one = torch.ones(max(M, N), device="cuda")
    y = blank(M, N, torch.float32)
    q8.cpdp_q8_matmul(a, one[:M], b, one[:N], y)
    assert bool((y == float(128 * 128 * K)).all())


def test_product_of_a_row_that_is_not_finite(q8):
    M, N, K = 70, 90, 256
    g = gen(5)
    a, b = put(ints(g, M, K), torch.int8), put(ints(g, N, K), torch.int8)
    sa, sb = torch.ones(M, device="cuda"), torch.ones(N, device="cuda")
    sa[3], sb[7] = math.nan, math.nan
    y = blank(M, N, torch.float32)
    q8.cpdp_q8_matmul(a, sa, b, sb, y)
    bad = torch.isnan(y)
    assert bool(bad[3].all()) and bool(bad[:, 7].all()) and int(bad.sum()) == M + N - 1


def act_64(kind, g, u):
    if kind == "gelu":
        return g * 0.5 * torch.erfc(-g / math.sqrt(2.0))
    return g * torch.sigmoid(g) * u


def act_bwd_64(kind, da, G, Uv):
    if kind == "gelu":
        return da * (0.5 * torch.erfc(-G / math.sqrt(2.0)) +
                     G * torch.exp(-G * G / 2) / math.sqrt(2 * math.pi)), None
    s = torch.sigmoid(G)
    return da * Uv * s * (1 + G * (1 - s)), da * G * s


@pytest.mark.parametrize("T,F", [(1, 1), (3, 9), (5, 513), (4, 1025), (7, 2049), (3, 4100),
                                 (3, 8200), (2, 16390), (2, 32770), (1100, 700), (1030, 1300)])
@pytest.mark.parametrize("kind", ["gelu", "swiglu"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_act_and_its_backward(q8, T, F, kind, dt):
    gen_ = gen(T + F)
    gated = kind == "swiglu"
    g = put(3 * randn(gen_, T, F), DT[dt], 5)
    u = put(randn(gen_, T, F), DT[dt], 5) if gated else None
    q, cg = blank(T, F, torch.int8), blank(T, F, torch.int8, 3)
    cu = blank(T, F, torch.int8, 3) if gated else None
    y = blank(T, F, torch.bfloat16)
    s, sg, su = (torch.empty(T, device="cuda") for _ in range(3))
    su = su if gated else None
    q8.cpdp_q8_act(kind, g, u, q=q, scale=s, y=y, cg=cg, sg=sg, cu=cu, su=su)
    a = act_64(kind, g.double(), u.double() if gated else None)
    # exp, reciprocal, erf and a few products: an absolute error for GELU, whose
    # 1 + erf cancels for negative g
    slack = 32 * U
    amax = a.abs().amax(1)
    assert bool((127 * s.double() >= amax * (1 - slack)).all())
    assert float((q.double() - a / s.double()[:, None]).abs().max()) <= 0.5 + 128 * slack
    assert torch.equal(y, (q.float() * s[:, None]).to(torch.bfloat16))
    for x, c, sc in ((g, cg, sg), (u, cu, su)):
        if x is not None:
            want = row_scale(x)
            assert torch.equal(sc.double(), want)
            assert float((c.double() - x.double() / want[:, None]).abs().max()) <= 0.5 + 127 * U
            untouched(c)
    untouched(q, y)

    da = put(randn(gen_, T, F), DT[dt])
    dg, du = blank(T, F, DT[dt], 1), blank(T, F, DT[dt], 1) if gated else None
    q8.cpdp_q8_act_bwd(kind, da, cg, sg, dg, cu=cu, su=su, du=du)
    G = cg.double() * sg.double()[:, None]
    Uv = cu.double() * su.double()[:, None] if gated else None
    want_g, want_u = act_bwd_64(kind, da.double(), G, Uv)
    # |G| 2^-24 from the exponent's argument, then a few roundings
    size = da.double().abs() * (Uv.abs() if gated else 1.0) * (1 + G.abs())
    over = B * want_g.abs() if dt == "bf16" else 0
    assert bool(((dg.double() - want_g).abs() <= 32 * U * size + over + 1e-37).all())
    if gated:
        size = da.double().abs() * G.abs() * (1 + G.abs())
        over = B * want_u.abs() if dt == "bf16" else 0
        assert bool(((du.double() - want_u).abs() <= 32 * U * size + over + 1e-37).all())
        untouched(du)
    untouched(dg)


def test_act_without_checkpoint_and_fused_halves(q8):
    """Serving keeps no checkpoint; g and u, and their gradients, may be the two
    halves of one matrix."""
    T, F = 33, 640
    z = put(randn(gen(6), T, 2 * F), torch.bfloat16)
    one, two = [], []
    for g, u, out in ((z[:, :F], z[:, F:], one),
                      (put(z[:, :F], torch.bfloat16), put(z[:, F:], torch.bfloat16), two)):
        q, s = blank(T, F, torch.int8), torch.empty(T, device="cuda")
        q8.cpdp_q8_act("swiglu", g, u, q=q, scale=s)
        out += [q.clone(), s]
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])
    cg, cu = ints(gen(7), T, F), ints(gen(8), T, F)
    sg, su = torch.rand(T, device="cuda"), torch.rand(T, device="cuda")
    da = put(randn(gen(9), T, F), torch.bfloat16)
    dz = torch.empty((T, 2 * F), dtype=torch.bfloat16, device="cuda")
    q8.cpdp_q8_act_bwd("swiglu", da, cg, sg, dz[:, :F], cu=cu, su=su, du=dz[:, F:])
    dg, du = (torch.empty((T, F), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q8.cpdp_q8_act_bwd("swiglu", da, cg, sg, dg, cu=cu, su=su, du=du)
    assert torch.equal(dz, torch.cat([dg, du], 1))


def test_act_rows_that_are_not_finite(q8):
    T, F = 4, 520
    g, u = randn(gen(10), T, F), randn(gen(11), T, F)
    g[0, 1], u[1, 519] = math.nan, math.inf
    g[2] = 0
    g, u = put(g, torch.float32), put(u, torch.float32)
    q, cg, cu = (blank(T, F, torch.int8) for _ in range(3))
    s, sg, su = (torch.empty(T, device="cuda") for _ in range(3))
    q8.cpdp_q8_act("swiglu", g, u, q=q, scale=s, cg=cg, sg=sg, cu=cu, su=su)
    assert torch.isnan(s).tolist() == [True, True, False, False]
    assert torch.isnan(sg).tolist() == [True, False, False, False]
    assert torch.isnan(su).tolist() == [False, True, False, False]
    assert bool((q[:3] == 0).all()) and float(s[2]) == SMALLEST


@pytest.mark.parametrize("kind", ["gelu", "swiglu"])
def test_act_bwd_against_differences(q8, kind):
    T, F, step = 9, 300, 1e-5
    g = gen(12)
    cg, cu = ints(g, T, F), ints(g, T, F)
    cg, cu = put(cg, torch.int8), put(cu, torch.int8)
    sg, su = torch.full((T,), 0.03125, device="cuda"), torch.full((T,), 0.0078125, device="cuda")
    da = put(randn(g, T, F), torch.float32)
    gated = kind == "swiglu"
    dg, du = blank(T, F, torch.float32), blank(T, F, torch.float32)
    q8.cpdp_q8_act_bwd(kind, da, cg, sg, dg, cu=cu if gated else None, su=su if gated else None,
                       du=du if gated else None)
    G, Uv = cg.double() * sg.double()[:, None], cu.double() * su.double()[:, None]
    by = (act_64(kind, G + step, Uv) - act_64(kind, G - step, Uv)) / (2 * step) * da.double()
    assert float((dg.double() - by).abs().max()) <= 1e-5 * float(da.abs().max())
    if gated:
        by = (act_64(kind, G, Uv + step) - act_64(kind, G, Uv - step)) / (2 * step) * da.double()
        assert float((du.double() - by).abs().max()) <= 1e-5 * float(da.abs().max())


GRADS = [(1, 1, 1), (1, 64, 8), (3, 100, 33), (64, 64, 64), (65, 127, 200), (197, 384, 387),
         (1000, 72, 515), (70, 1536, 384), (1576, 384, 130), (2048, 1000, 900),
         (700, 2048, 2300)]


@pytest.mark.parametrize("T,N,K", GRADS)
@pytest.mark.parametrize("dy_dt,out_dt", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"),
                                          ("f32", "bf16")])
def test_grads_of_a_product(q8, T, N, K, dy_dt, out_dt):
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
    # bf16: one rounding in the sum, one of the result
    tol = 2e-6 if out_dt == "f32" else math.sqrt(2.0 / 3.0) * B
    assert rel(dx, want_x) <= tol and rel(dw, want_w) <= tol
    untouched(dx, dw)


def test_grads_are_the_product_s_derivative(q8):
    """y = a b^T is linear in both: its change along a direction is the
    gradients' product with it."""
    T, N, K = 50, 70, 90
    g = gen(13)
    a, b = put(ints(g, T, K), torch.int8), put(ints(g, N, K), torch.int8)
    sa, sb = torch.rand(T, device="cuda"), torch.rand(N, device="cuda")
    dy = put(randn(g, T, N), torch.float32)
    dx, dw = blank(T, K, torch.float32), blank(N, K, torch.float32)
    q8.cpdp_q8_grad_input(dy, b, sb, dx)
    q8.cpdp_q8_grad_weight(dy, a, sa, dw)
    A, Bv = a.double() * sa.double()[:, None], b.double() * sb.double()[:, None]
    dA, dB = randn(g, T, K).double(), randn(g, N, K).double()
    loss = lambda x, w: float((dy.double() * (x @ w.t().contiguous())).sum())  # noqa: E731
    step = 1e-3
    by = (loss(A + step * dA, Bv) - loss(A - step * dA, Bv)) / (2 * step)
    assert abs(by - float((dx.double() * dA).sum())) <= 1e-5 * float(dx.norm()) * float(dA.norm())
    by = (loss(A, Bv + step * dB) - loss(A, Bv - step * dB)) / (2 * step)
    assert abs(by - float((dw.double() * dB).sum())) <= 1e-5 * float(dw.norm()) * float(dB.norm())


def test_grads_with_values_at_the_ends(q8):
    """Infinities and NaN in dy, dy near fp32's largest number, and 8-bit rows
    that were not finite, reach what depends on them and nothing else."""
    T, N, K = 70, 66, 80
    g = gen(14)
    a, b = put(ints(g, T, K), torch.int8), put(ints(g, N, K), torch.int8)
    a[:, 0], b[:, 0] = 1, 1
    sa, sb = torch.ones(T, device="cuda"), torch.ones(N, device="cuda")
    for dt in (torch.float32, torch.bfloat16):
        dy = randn(g, T, N)
        dy[2, 3], dy[4, 5] = math.inf, math.nan
        dy = put(dy, dt)
        dx, dw = blank(T, K, torch.float32), blank(N, K, torch.float32)
        q8.cpdp_q8_grad_input(dy, b, sb, dx)
        q8.cpdp_q8_grad_weight(dy, a, sa, dw)
        fine_x, fine_w = torch.isfinite(dx), torch.isfinite(dw)
        rows = torch.arange(T, device="cuda")
        assert bool(fine_x[(rows != 2) & (rows != 4)].all())
        assert float(dx[2, 0]) == math.inf and bool(torch.isnan(dx[4]).all())
        chans = torch.arange(N, device="cuda")
        assert bool(fine_w[(chans != 3) & (chans != 5)].all())
        assert float(dw[3, 0]) == math.inf and bool(torch.isnan(dw[5]).all())
    dy = torch.zeros(T, N, device="cuda")
    dy[1, 1] = 3.4e38  # rounds past the largest bfloat16
    dx = blank(T, K, torch.float32)
    q8.cpdp_q8_grad_input(put(dy, torch.float32), b, sb, dx)
    assert abs(float(dx[1, 0]) / 3.4e38 - 1) <= 4 * U
    sa[9] = math.nan
    q8.cpdp_q8_grad_weight(put(randn(g, T, N), torch.bfloat16), a, sa, dw)
    assert bool(torch.isnan(dw).all())


def test_nothing_to_do(q8):
    """No rows: nothing is written, but a gradient summed over none is zero."""
    z = lambda r, c, dt=torch.bfloat16: q8.empty_rows(r, c, dt)  # noqa: E731
    D, N = 40, 24
    e = torch.empty(0, device="cuda")
    w = torch.ones(D, device="cuda")
    q8.cpdp_q8_rows(z(0, D), z(0, D, torch.int8), e)
    q8.cpdp_q8_values(z(0, D, torch.int8), e, z(0, D))
    q8.cpdp_q8_norm(z(0, D), w, 1e-6, q=z(0, D, torch.int8), scale=e)
    dw = torch.full((D,), 5.0, device="cuda")
    q8.cpdp_q8_norm_bwd(z(0, D), z(0, D), w, e, z(0, D), dw)
    assert bool((dw == 0).all())
    q8.cpdp_q8_act("gelu", z(0, D), q=z(0, D, torch.int8), scale=e)
    q8.cpdp_q8_act_bwd("gelu", z(0, D), z(0, D, torch.int8), e, z(0, D))
    b, sb = z(N, D, torch.int8), torch.ones(N, device="cuda")
    q8.cpdp_q8_matmul(z(0, D, torch.int8), e, b, sb, z(0, N))
    q8.cpdp_q8_matmul(b, sb, z(0, D, torch.int8), e, z(N, 0))
    q8.cpdp_q8_grad_input(z(0, N), b, sb, z(0, D))
    for dt in (torch.float32, torch.bfloat16):
        g = blank(N, 37, dt, 5)
        g += 1
        q8.cpdp_q8_grad_weight(z(0, N), z(0, 37, torch.int8), e, g)
        assert bool((g == 0).all())
        untouched_by = padding(g).float()
        assert bool((untouched_by == 77).all())
    dx = z(9, D)
    dx.fill_(3)
    q8.cpdp_q8_grad_input(z(9, 0), z(0, D, torch.int8), e, dx)
    assert bool((dx == 0).all())


def layer_pass(q8, st):
    q8.cpdp_q8_norm(st["x"], st["w"], 1e-6, q=st["q"], scale=st["s"], residual=st["r"], h=st["h"],
                    rstd=st["rstd"])
    q8.cpdp_q8_matmul(st["q"], st["s"], st["b"], st["sb"], st["z"], workspace=st["ws"])
    q8.cpdp_q8_act("gelu", st["z"], q=st["qa"], scale=st["sa"], cg=st["cg"], sg=st["sg"])
    q8.cpdp_q8_act_bwd("gelu", st["dz"], st["cg"], st["sg"], st["dg"])
    q8.cpdp_q8_grad_input(st["dg"], st["b"], st["sb"], st["dq"], workspace=st["ws"])
    q8.cpdp_q8_grad_weight(st["dg"], st["q"], st["s"], st["db"], workspace=st["ws"])
    q8.cpdp_q8_norm_bwd(st["dq"], st["h"], st["w"], st["rstd"], st["dx"], st["dw"],
                        workspace=st["ws"])


def layer_state(q8, T=130, D=200, F=300):
    g = gen(20)
    e = q8.empty_rows
    st = {"x": put(randn(g, T, D), torch.bfloat16), "r": put(randn(g, T, D), torch.bfloat16),
          "w": 1 + 0.1 * randn(g, D), "b": put(ints(g, F, D), torch.int8),
          "sb": torch.rand(F, generator=g, device="cuda") / D,
          "dz": put(randn(g, T, F), torch.bfloat16)}
    st.update(h=e(T, D, torch.bfloat16), q=e(T, D, torch.int8), z=e(T, F, torch.bfloat16),
              qa=e(T, F, torch.int8), cg=e(T, F, torch.int8), dg=e(T, F, torch.bfloat16),
              dq=e(T, D, torch.bfloat16), db=e(F, D, torch.float32), dx=e(T, D, torch.bfloat16),
              dw=torch.empty(D, device="cuda"))
    for k in ("s", "rstd", "sa", "sg"):
        st[k] = torch.empty(T, device="cuda")
    st["ws"] = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    return st


OUT = ("h", "q", "s", "rstd", "z", "qa", "sa", "cg", "sg", "dg", "dq", "db", "dx", "dw")


def test_side_stream_and_reproducibility(q8):
    st = layer_state(q8)
    layer_pass(q8, st)
    torch.cuda.synchronize()
    first = {k: st[k].clone() for k in OUT}
    s = torch.cuda.Stream()
    for k in OUT:
        st[k].zero_()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        layer_pass(q8, st)
    s.synchronize()
    for k in OUT:
        assert torch.equal(st[k], first[k]), k


def test_captured_graph(q8):
    st = layer_state(q8)
    layer_pass(q8, st)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        layer_pass(q8, st)
    for k in range(4):
        st["x"].add_(0.25)
        st["dz"].mul_(1.5)
        layer_pass(q8, st)
        torch.cuda.synchronize()
        eager = {k2: st[k2].clone() for k2 in OUT}
        for k2 in OUT:
            st[k2].zero_()
        st["ws"].fill_(255)
        g.replay()
        torch.cuda.synchronize()
        for k2 in OUT:
            assert torch.equal(st[k2], eager[k2]), (k, k2)


def test_a_stream_that_is_given_needs_a_workspace(q8):
    st = layer_state(q8)
    s = torch.cuda.Stream()
    with pytest.raises(ValueError, match="workspace"):
        q8.cpdp_q8_norm_bwd(st["x"], st["h"], st["w"], st["rstd"], st["dx"], st["dw"], stream=s)
    s.wait_stream(torch.cuda.current_stream())
    q8.cpdp_q8_norm_bwd(st["x"], st["r"], st["w"], st["rstd"].fill_(1), st["dx"], st["dw"],
                        workspace=st["ws"], stream=s)
    s.synchronize()


def test_offsets_past_32_bits(q8):
    """Matrices of more than 2^32 bytes: the last rows are right."""
    T, D = 600_001, 4096
    x = torch.empty((T, D), dtype=torch.bfloat16, device="cuda")
    x.fill_(0.5)
    tail = randn(gen(30), 3, D)
    x[-3:] = tail.to(torch.bfloat16)
    q, s = torch.empty((T, D), dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    y = torch.empty((T, D), dtype=torch.bfloat16, device="cuda")
    q8.cpdp_q8_rows(x, q, s, y=y)
    want = row_scale(x[-3:])
    assert torch.equal(s[-3:].double(), want)
    assert torch.equal(q[-3:].double(), torch.round(x[-3:].double() / want[:, None]))
    assert torch.equal(y[-3:], (q[-3:].float() * s[-3:, None]).to(torch.bfloat16))
    # a product whose operand and result are both that large
    w = torch.zeros((4096, D), dtype=torch.int8, device="cuda")
    w[:, 1], w[5, 2] = 1, 3
    one = torch.ones(4096, device="cuda")
    q8.cpdp_q8_matmul(q, s, w, one, y)
    assert torch.equal(y[-3:, 0], (q[-3:, 1].float() * s[-3:]).to(torch.bfloat16))
    both = q[-3:, 1].float() + 3 * q[-3:, 2].float()
    assert torch.equal(y[-3:, 5], (both * s[-3:]).to(torch.bfloat16))


def test_refusals(q8):
    T, D = 8, 32
    x = q8.empty_rows(T, D, torch.bfloat16)
    q, s = q8.empty_rows(T, D, torch.int8), torch.empty(T, device="cuda")
    from paper_2607_21224_amd import cpdp
    with pytest.raises(ValueError, match="x"):
        q8.cpdp_q8_rows(x.half(), q, s)
    with pytest.raises(ValueError, match="q"):
        q8.cpdp_q8_rows(x, q[:, :31], s)
    with pytest.raises(ValueError, match="scale"):
        q8.cpdp_q8_rows(x, q, s[:7])
    with pytest.raises(ValueError, match="dense"):
        q8.cpdp_q8_rows(x[:, ::2], q[:, :16], s)
    with pytest.raises(ValueError, match="current GPU"):
        q8.cpdp_q8_rows(x.cpu(), q, s)
    with pytest.raises(cpdp.CpdpError) as e:  # rows that start on odd addresses
        q8.cpdp_q8_rows(torch.empty((T, 33), dtype=torch.bfloat16, device="cuda"),
                        q8.empty_rows(T, 33, torch.int8), s)
    assert e.value.status == cpdp.CPDP_ERR_MISALIGNED
    with pytest.raises(cpdp.CpdpError) as e:
        q8.cpdp_q8_norm(x, torch.ones(D, device="cuda"), -1.0, q=q, scale=s)
    assert e.value.status == cpdp.CPDP_ERR_INVALID_ARG
    with pytest.raises(cpdp.CpdpError) as e:  # a residual without a place for the sum
        q8.cpdp_q8_norm(x, torch.ones(D, device="cuda"), 0.0, q=q, scale=s, residual=x.clone())
    assert e.value.status == cpdp.CPDP_ERR_NULL
    with pytest.raises(ValueError, match="kind"):
        q8.cpdp_q8_act("relu", x, q=q, scale=s)
    with pytest.raises(ValueError, match="u"):
        q8.cpdp_q8_act("swiglu", x, q=q, scale=s)
    wide = torch.zeros((2, 131088), dtype=torch.int8, device="cuda")
    with pytest.raises(cpdp.CpdpError) as e:
        q8.cpdp_q8_matmul(wide, s[:2], wide, s[:2], torch.empty((2, 8), device="cuda")[:, :2])
    assert e.value.status == cpdp.CPDP_ERR_INVALID_ARG
