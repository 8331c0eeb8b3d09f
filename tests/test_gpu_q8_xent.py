"""The loss on 8-bit rows and its gradients against their definitions in 64 bits, and the
gradients against differences of the loss.

Tolerances, with u = 2^-24 and b = 2^-8.  Z is the largest |z| of a token, L a bound on
the fp32 additions that one term of a token's sum passes through, and e = 4 u the error
of exp and log.
* z: the exact sum converted and scaled, 3 roundings: 3 u |z|.
* lse: 3 u Z from the logits, (L + 4) u + e from the sum (all of it positive; exp's argument
  is rounded: 2 Z u more, and scaled to a power of two: Z u twice), u |lse| for the last
  addition.  loss: that, 3 u |z| of the target and u |loss|.
* p = exp(z - lse): 3 u Z + lse's error + 3 u (Z + |lse|) + e, relative: call it r.
  d = g (p - 1?): |g| (p r + 3 u (p + 1?)).
* dx, dw: R u of the terms' sizes for R additions in any order, 4 u for scaling, the terms'
  own errors, and what the numbers that hold a term leave out: h = 2^-11, half a step of
  fp16, once for a bf16 result, squared for an fp32 one; and half the smallest fp16 number,
  2^-25, where the largest scale, M, is brought to 2^14 or more: 2^-39 M |q| for each term,
  2^-51 M |q| for an fp32 result, whose second number is held 2^12 times as large.  M is the
  largest |g x_scale| for dw and, times the row's |g|, the largest |w_scale| for dx.
  Up to 64 tokens: b for terms that are rounded to one bfloat16 number, and for what falls
  below the smallest normal one, 2^-126, which the matrix cores take as 0, up to three
  parts' worth, the first of them the largest: 2^-125 in all, for each term and times |q|.
  b for a bf16 result's own rounding.
"""
import math

import pytest
import torch

import xent_sizes
from test_gpu_q8 import B, U, blank, gen, ints, put, q8, randn, rel, untouched  # noqa: F401
from xent_sizes import BF16, NONE

pytestmark = pytest.mark.gpu

DTYPE = (torch.float32, torch.bfloat16)
E = 4 * U
H = 2.0 ** -11


class Case:
    """Random 8-bit rows whose logits are a few units, targets that rows lean towards, and
    the definitions in 64 bits."""

    def __init__(self, T, V, K, seed=0, size=2.5, ignored=0.1):
        g = gen(T + V + K + seed)
        self.T, self.V, self.K = T, V, K
        self.x, self.w = put(ints(g, T, K), torch.int8, 7), put(ints(g, V, K), torch.int8, 21)
        rand = lambda *s: torch.rand(s, generator=g, device="cuda")  # noqa: E731
        self.target = (V * rand(T)).long().clamp_max(V - 1)
        lean = rand(T) < 0.4
        rows = self.w[self.target[lean]]
        mix = rand(len(rows), K) < rand(len(rows), 1)
        self.x[lean] = torch.where(mix, rows, self.x[lean])
        root = math.sqrt(size / (5300 * math.sqrt(K)))
        self.xs = root * torch.exp(0.3 * randn(g, T))
        self.ws = (root * torch.exp(0.3 * randn(g, V))).to(torch.bfloat16).float()
        self.g = randn(g, T) / T
        skip = rand(T) < ignored
        self.target[skip] = torch.where(rand(int(skip.sum())) < 0.5, -100, -1)
        self.g[skip] = float("nan")
        self.counts = self.target >= 0

    def held(self):
        return self.x, self.xs, self.w, self.ws, self.target

    def forward(self, q8, **kw):  # noqa: F811
        loss, lse = (torch.full((self.T + 1,), 77.0, device="cuda") for _ in range(2))
        q8.cpdp_q8_xent(*self.held(), loss[:-1], lse[:-1], **kw)
        assert loss[-1] == lse[-1] == 77
        return loss[:-1], lse[:-1]

    def backward(self, q8, lse, dx_dt, dw_dt, **kw):  # noqa: F811
        dx = blank(self.T, self.K, DTYPE[dx_dt], 5) if dx_dt != NONE else None
        dw = blank(self.V, self.K, DTYPE[dw_dt], 3) if dw_dt != NONE else None
        q8.cpdp_q8_xent_bwd(*self.held(), lse, self.g, dx, dw, **kw)
        untouched(*[v for v in (dx, dw) if v is not None])
        return dx, dw

    def logits(self):
        """z, and the most that an fp32 sum of exp's may be off, relative."""
        z = torch.mm(self.x.double(), self.w.double().t().contiguous())
        return z * self.xs.double()[:, None] * self.ws.double()

    def check_forward(self, loss, lse):
        z = self.logits()
        want = torch.logsumexp(z, 1)
        top = z.abs().amax(1)
        L = self.V / 256 + 64
        off = 6 * U * top + (L + 4) * U + E + U * want.abs()
        assert bool(((lse.double() - want).abs() <= off).all())
        self.lse_off = off
        hit = z.gather(1, self.target.clamp_min(0)[:, None])[:, 0]
        want = torch.where(self.counts, want - hit, 0.0)
        off = torch.where(self.counts, off + 3 * U * hit.abs() + U * want.abs(), 0.0)
        assert bool(((loss.double() - want).abs() <= off).all())

    def gradients(self):
        """d with its error, in 64 bits, zero where tokens do not count."""
        z = self.logits()
        lse = torch.logsumexp(z, 1, keepdim=True)
        p = torch.exp(z - lse)
        top = z.abs().amax(1, keepdim=True)
        r = 6 * U * (top + lse.abs()) + self.lse_off[:, None] + E
        g = torch.where(self.counts, self.g.double(), 0.0)[:, None]
        hot = torch.zeros_like(p)
        hot.scatter_(1, self.target.clamp_min(0)[:, None], 1.0)
        return g * (p - hot), g.abs() * (p * r + 3 * U * (p + hot))

    def check(self, got, d, off, q, scale, largest, dt):
        """got against d (scale q), d known up to off; largest: M, for each row."""
        R, right = d.shape[1], q.double() * scale.double()[:, None]
        want, size = torch.mm(d, right), torch.mm(d.abs(), right.abs())
        bf16 = dt == BF16
        if self.T > 64:
            held = H if bf16 else H * H
            floor = 2.0 ** (-39 if bf16 else -51) * largest[:, None]
        else:
            held, floor = B if bf16 else 0.0, 2.0 ** -125
        slack = torch.mm(off, right.abs()) + (held + (R + 4) * U) * size
        slack = slack + floor * q.double().abs().sum(0)
        if bf16:
            slack = slack + B * (want.abs() + slack)
        off = (got.double() - want).abs()
        bad = (~(off <= slack + 1e-37)).nonzero()
        assert len(bad) == 0, (len(bad), [(i, float(got[i]), float(want[i]), float(slack[i]))
                                          for i in map(tuple, bad[:3].tolist())])

    def check_backward(self, dx, dw, dx_dt, dw_dt):
        d, off = self.gradients()
        g = torch.where(self.counts, self.g.double(), 0.0).abs()
        if dx_dt != NONE:
            self.check(dx, d, off, self.w, self.ws, g * self.ws.double().abs().max(), dx_dt)
            assert not dx[~self.counts].any()
        if dw_dt != NONE:
            largest = (g * self.xs.double().abs()).max().expand(self.V)
            self.check(dw, d.t().contiguous(), off.t().contiguous(), self.x, self.xs, largest,
                       dw_dt)


@pytest.mark.parametrize("T,V,K", xent_sizes.SMALL + xent_sizes.MIDDLE + xent_sizes.LARGE)
def test_loss(q8, T, V, K):  # noqa: F811
    c = Case(T, V, K)
    loss, lse = c.forward(q8)
    c.check_forward(loss, lse)
    again = c.forward(q8)
    assert torch.equal(again[0], loss) and torch.equal(again[1], lse)


@pytest.mark.parametrize("types", xent_sizes.TYPES)
@pytest.mark.parametrize("T,V,K", xent_sizes.SMALL + xent_sizes.MIDDLE + xent_sizes.LARGE)
def test_gradients(q8, T, V, K, types):  # noqa: F811
    c = Case(T, V, K)
    loss, lse = c.forward(q8)
    c.check_forward(loss, lse)
    got = c.backward(q8, lse, *types)
    c.check_backward(*got, *types)
    again = c.backward(q8, lse, *types)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("T,V,K", xent_sizes.ONE)
@pytest.mark.parametrize("types", xent_sizes.ALONE)
def test_one_gradient_alone(q8, T, V, K, types):  # noqa: F811
    c = Case(T, V, K)
    lse = c.forward(q8)[1]
    c.check_forward(c.forward(q8)[0], lse)
    c.check_backward(*c.backward(q8, lse, *types), *types)


@pytest.mark.parametrize("T,V,K", [(3, 100, 64), (70, 300, 130), (500, 3001, 70)])
def test_against_differences(q8, T, V, K):  # noqa: F811
    """The loss' derivative by log x_scale is sum_k dx x x_scale.  A central difference of step
    h is off by h^2 / 6 of the third derivative, the third cumulant of a token's logits and so
    at most R^3 for logits in a range of R, and by the loss' own error over h."""
    c = Case(T, V, K, ignored=0.0)
    c.g = torch.ones(T, device="cuda")
    loss, lse = c.forward(q8)
    dx, _ = c.backward(q8, lse, 0, 0)
    scale, h, at = c.xs, 2.0 ** -9, []
    for s in (1 + h, 1 - h):
        c.xs = scale * s
        at.append((c.forward(q8)[0].double(), torch.log(c.xs.double() / scale.double())))
    c.xs = scale
    slope = (at[0][0] - at[1][0]) / (at[0][1] - at[1][1])
    z = c.logits()
    R = z.amax(1) - z.amin(1)
    got = (dx.double() * c.x.double() * scale.double()[:, None]).sum(1)
    noise = (20 * U * z.abs().amax(1) + (V / 256 + 80) * U) / h
    # (exp(h) is not quite 1 + h: the second derivative, at most R^2, times h^2)
    assert bool(((got - slope).abs() <= (R ** 3 + 6 * R ** 2) * h * h / 6 + noise).all())


@pytest.mark.parametrize("T", [1, 40, 300])
def test_tokens_that_do_not_count(q8, T):  # noqa: F811
    """All of them, then some whose rows are not finite."""
    c = Case(T, 515, 100, ignored=1.1)
    loss, lse = c.forward(q8)
    assert not loss.any() and bool(lse.isfinite().all())
    for types in xent_sizes.TYPES:
        dx, dw = c.backward(q8, lse, *types)
        assert not dx.any() and not dw.any()
    c = Case(T + 1, 515, 100, ignored=0.0)
    ref = Case(T + 1, 515, 100, ignored=0.0)
    for k, bad in enumerate([float("nan"), float("inf"), -float("inf")]):
        i = k * (T // 3)
        c.target[i] = ref.target[i] = -1 - k
        c.xs[i], c.g[i] = bad, bad
    want, got = ref.forward(q8), c.forward(q8)
    assert torch.equal(want[0], got[0]) and bool((got[0][c.target < 0] == 0).all())
    for types in xent_sizes.TYPES:
        a, b = ref.backward(q8, want[1], *types), c.backward(q8, got[1], *types)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("T", [5, 80, 300])
def test_a_token_that_is_not_finite(q8, T):  # noqa: F811
    c = Case(T, 400, 64, ignored=0.0)
    ref = c.forward(q8)
    dx_ref = c.backward(q8, ref[1], 0, 0)[0]
    scale, target = c.xs[2].clone(), c.target[2].clone()
    for change in ("scale", "past the classes", "far past"):
        if change == "scale":
            c.xs[2] = float("nan")
        else:
            c.xs[2], c.target[2] = scale, c.V if change == "past the classes" else 1 << 40
        loss, lse = c.forward(q8)
        assert loss[2].isnan()
        others = torch.arange(T, device="cuda") != 2
        assert torch.equal(loss[others], ref[0][others])
        for types in xent_sizes.TYPES:
            dx, dw = c.backward(q8, lse, *types)
            assert bool(dx[2].isnan().all()) and bool(dw.isnan().all())
            if types[0] != BF16:
                assert torch.equal(dx[others], dx_ref[others])
    c.target[2] = target
    # a class that is not finite is part of every token's sum
    c.ws[7] = float("nan")
    assert bool(c.forward(q8)[0].isnan().all())


@pytest.mark.parametrize("T", [3, 100])
def test_steep_and_flat_logits(q8, T):  # noqa: F811
    # logits of +-10^4: exp overflows anywhere but at the row's maximum
    c = Case(T, 700, 128, size=4000.0, ignored=0.0)
    loss, lse = c.forward(q8)
    c.check_forward(loss, lse)
    c.check_backward(*c.backward(q8, lse, 0, 0), 0, 0)
    # all alike
    c.ws.zero_()
    loss, lse = c.forward(q8)
    assert bool(((loss.double() - math.log(700)).abs() <= 8 * U * 10).all())
    dx, dw = c.backward(q8, lse, 0, 0)
    assert not dx.any()
    c.check_forward(loss, lse)
    c.check_backward(dx, dw, 0, 0)
    # nothing but one class
    c = Case(T, 1, 128)
    loss, lse = c.forward(q8)
    assert not loss.any()
    dx, dw = c.backward(q8, lse, 0, 0)
    off = float((c.xs[c.counts] * c.g[c.counts]).abs().sum()) * 127 * 16 * U
    assert float(dw.abs().max()) <= off


@pytest.mark.parametrize("types", xent_sizes.TYPES)
@pytest.mark.parametrize("T", [5, 100, 700])
def test_small_probabilities(q8, T, types):  # noqa: F811
    """Half of the classes have logits some 15 to 70 below the others'."""
    c = Case(T, 700, 128, size=6.0)
    c.x[:, :32], c.w[1::2, :32], c.w[::2, :32] = 100, -100, 0
    loss, lse = c.forward(q8)
    c.check_forward(loss, lse)
    c.check_backward(*c.backward(q8, lse, *types), *types)


@pytest.mark.parametrize("scale", [2.0 ** -100, 2.0 ** -30, 2.0 ** 60])
def test_weights_of_any_size(q8, scale):  # noqa: F811
    """Tokens' weights of very small and large sizes scale the gradients and nothing else."""
    c = Case(100, 700, 128, ignored=0.0)
    lse = c.forward(q8)[1]
    c.g.uniform_(0.5, 1.0)
    want = c.backward(q8, lse, 0, 0)
    c.g *= scale
    got = c.backward(q8, lse, 0, 0)
    for a, b in zip(want, got):
        normal = a.abs() * scale > 2.0 ** -125
        assert torch.equal((a * scale)[normal], b[normal])
        assert bool(((a * scale - b)[~normal].abs() <= 2.0 ** -125).all())


def test_logits_past_the_largest_number(q8):  # noqa: F811
    """One class' logit is -infinity (no probability), or +infinity (no loss)."""
    c = Case(70, 300, 16, ignored=0.0)
    c.x.fill_(1), c.w.fill_(1)
    c.xs.fill_(1.0), c.ws.fill_(0.01)
    c.target.fill_(5)
    c.w[9] = -1
    c.ws[9] = float("inf")
    loss, lse = c.forward(q8)
    assert bool(((loss.double() - math.log(299)).abs() <= 64 * U * 10).all())
    c.w[9] = 1
    assert bool(c.forward(q8)[0].isnan().all())


def test_no_tokens(q8):  # noqa: F811
    c = Case(4, 300, 70)
    for k in ("x", "xs", "target", "g"):
        setattr(c, k, getattr(c, k)[:0])
    c.T, c.counts = 0, c.counts[:0]
    loss, lse = c.forward(q8)
    for types in xent_sizes.TYPES:
        dx = torch.empty((0, 80), dtype=DTYPE[types[0]], device="cuda")[:, :70]
        dw = blank(300, 70, DTYPE[types[1]], 3).fill_(5)
        q8.cpdp_q8_xent_bwd(*c.held(), lse, c.g, dx, dw)
        assert not dw.any()
        untouched(dw)


def test_rows_past_32_bits(q8):  # noqa: F811
    """Weights and gradients of more than 2^31 elements: the last classes' logits and gradients
    lie past what 32 bits count."""
    T, V, K = 3, 70003, 32768
    free = torch.cuda.mem_get_info()[0]
    assert free > 40 << 30
    w = torch.zeros((V, K), dtype=torch.int8, device="cuda")
    w[V - 5:] = ints(gen(1), 5, K).to(torch.int8)
    x = ints(gen(2), T, K).to(torch.int8)
    xs, ws = torch.full((T,), 1e-5, device="cuda"), torch.full((V,), 1e-2, device="cuda")
    target = torch.tensor([V - 1, V - 3, 0], device="cuda")
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    q8.cpdp_q8_xent(x, xs, w, ws, target, loss, lse)
    z = torch.zeros((T, V), dtype=torch.float64, device="cuda")
    z[:, V - 5:] = torch.mm(x.double(), w[V - 5:].double().t().contiguous()) * 1e-7
    z = z * (xs[0].double() * ws[0].double() / 1e-7)
    want = torch.logsumexp(z, 1) - z.gather(1, target[:, None])[:, 0]
    assert bool(((loss.double() - want).abs() <= 2e-4).all())  # (V / 256 + 80) u and more
    dw = torch.empty((V, K), dtype=torch.bfloat16, device="cuda")
    g = torch.ones(T, device="cuda")
    q8.cpdp_q8_xent_bwd(x, xs, w, ws, target, lse, g, dw=dw)
    d = torch.softmax(z, 1)
    d[torch.arange(T), target] -= 1
    for rows in (slice(0, 3), slice(V - 5, V), slice(65534, 65540)):
        exact = torch.mm(d[:, rows].t().contiguous(), x.double() * xs.double()[:, None])
        size = torch.mm(d[:, rows].t().abs().contiguous(), x.double().abs() * xs.double()[:, None])
        assert bool(((dw[rows].double() - exact).abs() <= (2 * B + 3e-4) * size).all())


def test_slices_of_wider_matrices(q8):  # noqa: F811
    """Rows and results that are columns of wider matrices, as a model's tensors lie."""
    c = Case(70, 300, 64)
    loss, lse = c.forward(q8)
    dx, dw = c.backward(q8, lse, 1, 0)
    wide = torch.full((70, 256), 55, dtype=torch.int8, device="cuda")
    wide[:, 128:192] = c.x
    c.x = wide[:, 128:192]
    grads = torch.full((300, 200), 55.0, device="cuda")
    again = c.forward(q8)
    assert torch.equal(again[0], loss)
    out = torch.full((70, 96), 55.0, dtype=torch.bfloat16, device="cuda")
    q8.cpdp_q8_xent_bwd(*c.held(), lse, c.g, out[:, 16:80], grads[:, 100:164])
    assert torch.equal(out[:, 16:80], dx) and torch.equal(grads[:, 100:164], dw)
    assert bool((out[:, :16] == 55).all()) and bool((out[:, 80:] == 55).all())
    assert bool((grads[:, :100] == 55).all()) and bool((grads[:, 164:] == 55).all())


SIZES = [(9, 1001, 130), (128, 100, 384), (700, 9001, 130)]


@pytest.mark.parametrize("T,V,K", SIZES)
def test_captured(q8, T, V, K):  # noqa: F811
    """Two graphs that share a workspace, replayed in turn, with eager calls of other sizes in
    the same workspace between them."""
    cases = [Case(T, V, K, seed) for seed in (1, 2)]
    dts = DTYPE[1], DTYPE[0]
    need = max(q8.cpdp_q8_xent_workspace(T, V, K), q8.cpdp_q8_xent_bwd_workspace(T, V, K, *dts))
    ws = torch.empty(max(need, 1 << 24), dtype=torch.uint8, device="cuda")
    want = []
    for c in cases:
        loss, lse = c.forward(q8)
        want.append((loss, lse, *c.backward(q8, lse, 1, 0)))
    side, graphs, got = torch.cuda.Stream(), [], []
    torch.cuda.synchronize()
    for c in cases:
        out = [torch.empty(T, device="cuda"), torch.empty(T, device="cuda"),
               blank(T, K, dts[0]), blank(V, K, dts[1])]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            q8.cpdp_q8_xent(*c.held(), out[0], out[1], workspace=ws)
            q8.cpdp_q8_xent_bwd(*c.held(), out[1], c.g, out[2], out[3], workspace=ws)
        graphs.append(graph), got.append(out)
    other = Case(33, 77, 50)
    for _ in range(3):
        for k in (0, 1):
            for v in got[k]:
                v.fill_(3)
            graphs[k].replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got[k], want[k]))
            loss, lse = other.forward(q8, workspace=ws)
            other.backward(q8, lse, 0, 0, workspace=ws)
            other.check_forward(loss, lse)


def test_on_a_stream(q8):  # noqa: F811
    c = Case(200, 3001, 130)
    loss, lse = c.forward(q8)
    dx, dw = c.backward(q8, lse, 1, 1)
    s = torch.cuda.Stream()
    ws = torch.empty(q8.cpdp_q8_xent_bwd_workspace(200, 3001, 130, DTYPE[1], DTYPE[1]) + (1 << 22),
                     dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    for stream in (s, s.cuda_stream):
        again = c.forward(q8, stream=stream, workspace=ws)
        s.synchronize()
        assert torch.equal(again[0], loss)
    with torch.cuda.stream(s):
        a, b = c.backward(q8, lse, 1, 1)
    s.synchronize()
    assert torch.equal(a, dx) and torch.equal(b, dw)
    with pytest.raises(ValueError, match="workspace"):
        c.forward(q8, stream=s)


def test_refusals(q8):  # noqa: F811
    c = Case(6, 40, 32)
    loss, lse = c.forward(q8)
    x, xs, w, ws, target = c.held()
    for bad, what in ((target.int(), "int64"), (target[:5], "vector"), (target[None], "vector"),
                      (target.cpu(), "GPU")):
        with pytest.raises(ValueError, match=what):
            q8.cpdp_q8_xent(x, xs, w, ws, bad, loss, lse)
    with pytest.raises(ValueError, match="shape"):
        q8.cpdp_q8_xent(x, xs, w[:, :16], ws, target, loss, lse)
    with pytest.raises(ValueError, match="neither"):
        q8.cpdp_q8_xent_bwd(x, xs, w, ws, target, lse, c.g)
    with pytest.raises(ValueError, match="shape"):
        q8.cpdp_q8_xent_bwd(x, xs, w, ws, target, lse, c.g, dx=blank(5, 32, DTYPE[0]))
    with pytest.raises(ValueError, match="float32"):
        q8.cpdp_q8_xent_bwd(x, xs, w, ws, target, lse.bfloat16(), c.g, dx=blank(6, 32, DTYPE[0]))
