"""The loss of tokens whose target has nearly all of the probability, and its gradients, at
large logits that fp32 holds exactly: what is lost there is the operators' own.

Every class has the logit `base`, a whole number of 16ths, and a token's target one of base +
gap: with s = (V - 1) exp(-gap) its loss is log(1 + s), whatever base is.

Tolerance, with u = 2^-24.  An exponential's argument is rounded and scaled to a power of two by
a rounded constant, 2 gap u, and is itself within 4 u.  One term passes through A additions at
most: 9 of a lane's, 2 between lanes, 3 between wavefronts, and V / 1024 + 21 between tiles.
Those of sums of the others' alone are relative to s, those after the target's 1 to 1 + s, and a
product where parts are joined is as an addition.  So the sum is off by

    s (2 gap + 4 + 2 A) u + A (1 + s) u

at most, the loss by that over 1 + s, its logarithm 2 u of it, and the last addition u.
lse: the same, and u |lse| for its own rounding.
miss, 1 - exp(-loss): as the loss, and 2 u of it.
p of the others: lse's error and 2 (gap + loss) u + 4 u, relative.  d has that times |g|, the
target's the error of miss, and u for the product.  Without miss the target's is 1 - exp(z - lse):
lse's error, 2 loss u and 4 u.
"""
import math

import pytest
import torch

import xent_sizes
from test_gpu_q8 import U, q8  # noqa: F401
from test_gpu_q8_xent import Case

pytestmark = pytest.mark.gpu

GAP = 5.75  # and twice and three times that
SIZES = [(1, 33), (9, 700), (16, 5003), (40, 5003), (65, 700), (130, 33), (300, 5003)]


class Confident(Case):
    def __init__(self, T, V, base, K=40):
        self.T, self.V, self.K = T, V, K
        hot = min(V, K - 2)
        classes = torch.arange(hot, device="cuda") * (V // hot)
        t = torch.arange(T, device="cuda")
        self.target, more = classes[t % hot], 1 + t % 3
        ld = (K + 15) // 16 * 16
        x = torch.zeros((T, ld), dtype=torch.int8, device="cuda")
        w = torch.zeros((V, ld), dtype=torch.int8, device="cuda")
        # 64 x whole + rest = 16 base
        x[:, 0], x[:, 1] = 64, 1
        w[:, 0], w[:, 1] = int(16 * base) // 64, int(16 * base) % 64
        x[t, 2 + t % hot] = more.to(torch.int8)
        w[classes, 2 + torch.arange(hot, device="cuda")] = int(16 * GAP)
        self.x, self.w = x[:, :K], w[:, :K]
        self.xs = torch.full((T,), 0.25, device="cuda")
        self.ws = torch.full((V,), 0.25, device="cuda")
        self.gap = GAP * more.double()
        self.s = (V - 1) * torch.exp(-self.gap)
        self.top = base + self.gap
        A = 35 + V / 1024
        self.off = (self.s * (2 * self.gap + 4 + 2 * A) / (1 + self.s) + A) * U
        self.g = (1 + t % 5) / T
        self.counts = self.target >= 0
        self.with_miss = True

    def gradients(self):
        """d with its error: of the others p alike, of the target 1 less all of theirs."""
        loss = torch.log1p(self.s)[:, None]
        p = (1 / (torch.exp(self.gap) + self.V - 1))[:, None].expand(-1, self.V).clone()
        miss = (self.s / (1 + self.s))[:, None]
        lse_off = self.off[:, None] + 3 * U * loss + U * (loss + self.top[:, None])
        off = p * (lse_off + (2 * (self.gap[:, None] + loss) + 4) * U)
        hit = self.off[:, None] + (3 * loss + 2 * miss) * U
        if not self.with_miss:
            hit = lse_off + (2 * loss + 4) * U
        at = self.target[:, None]
        p.scatter_(1, at, -miss), off.scatter_(1, at, hit)
        g = self.g.double()[:, None]
        return g * p, g * (off + U * p.abs())


@pytest.mark.parametrize("base", [0, 50, 100, 300])
@pytest.mark.parametrize("T,V", SIZES)
def test_loss(q8, T, V, base):  # noqa: F811
    c = Confident(T, V, base)
    z = (c.x.double() @ c.w.double().t()) / 16
    assert torch.equal(z[torch.arange(T), c.target], c.top) and float(z.amin()) == base
    loss, lse = c.forward(q8)
    want = torch.log1p(c.s)
    bad = (loss.double() - want).abs() > c.off + 3 * U * want
    assert not bad.any(), (loss[bad][:3], want[bad][:3], c.off[bad][:3])
    want = want + c.top
    assert bool(((lse.double() - want).abs() <= c.off + 3 * U * torch.log1p(c.s) + U * want).all())


def test_the_loss_of_one_class_is_zero(q8):  # noqa: F811
    for T in (1, 40, 130):
        c = Confident(T, 1, 300)
        loss, lse = c.forward(q8)
        assert not loss.any() and torch.equal(lse.double(), c.top)


def test_a_target_that_has_no_probability(q8):  # noqa: F811
    """Its logit is -infinity: an infinite loss, as before; where all are, there is none."""
    for T in (1, 40, 130):
        c = Confident(T, 700, 50)
        c.w[c.target] = -1
        c.ws[c.target] = math.inf
        loss, lse = c.forward(q8)
        assert bool((loss == math.inf).all()) and bool(lse.isfinite().all())
        c.w.fill_(-1), c.ws.fill_(math.inf)
        loss, lse = c.forward(q8)
        assert bool(loss.isnan().all()) and bool((lse == -math.inf).all())


@pytest.mark.parametrize("types", [(0, 0), (1, 1)])
@pytest.mark.parametrize("base", [0, 50, 100, 300])
@pytest.mark.parametrize("T,V", SIZES)
def test_gradients(q8, T, V, base, types):  # noqa: F811
    """With miss, to the bounds above; without, to those that the header gives, |lse| 2^-24."""
    c = Confident(T, V, base)
    miss = torch.empty(T, device="cuda")
    loss, lse = c.forward(q8, miss=miss)
    want = c.s / (1 + c.s)
    assert bool(((miss.double() - want).abs() <= c.off + (3 * torch.log1p(c.s) + 2 * want) * U).all())
    assert all(torch.equal(a, b) for a, b in zip(c.forward(q8), (loss, lse)))
    c.check_backward(*c.backward(q8, lse, *types, miss=miss), *types)
    c.with_miss = False
    c.check_backward(*c.backward(q8, lse, *types), *types)


@pytest.mark.parametrize("T,V", SIZES)
def test_slopes_add_up_to_nothing(q8, T, V):  # noqa: F811
    """All classes have the same weights in two channels, and the sum of d over the classes is 0:
    with miss what is left of it there does not grow with the logits but as the others' p do."""
    c = Confident(T, V, 300)
    miss = torch.empty(T, device="cuda")
    loss, lse = c.forward(q8, miss=miss)
    dx = c.backward(q8, lse, 0, xent_sizes.NONE, miss=miss)[0][:, 0].double().abs()
    d, off = c.gradients()
    size = d.abs().sum(1)
    # (a floor of 2^-51 or less of the largest scale for each term, as in the other tests)
    room = off.sum(1) + ((V + 4) * U + 2.0 ** -22) * size + V * 2.0 ** -51 * c.g.double()
    assert bool((dx <= room * float(c.w[0, 0]) * 0.25).all())


@pytest.mark.parametrize("T", [1, 9, 40, 130])
def test_miss_of_tokens_without_one(q8, T):  # noqa: F811
    """A token that does not count has 0, one whose target is not there NaN, one whose target has
    no probability 1."""
    c = Confident(T, 700, 50)
    miss = torch.full((T + 1,), 7.0, device="cuda")
    for target, scale in ((-5, 0.25), (700, 0.25), (3, math.inf)):
        c.target.fill_(target)
        c.w[3], c.ws[3] = -1, scale
        c.forward(q8, miss=miss[:-1])
        got = miss[:-1]
        assert bool((got.isnan() if target == 700 else got == float(target == 3)).all())
    assert miss[-1] == 7


@pytest.mark.parametrize("T,V,K", [(9, 1001, 130), (63, 1000, 63), (128, 100, 384),
                                   (700, 9001, 130), (33, 300007, 40), (2100, 70001, 130)])
@pytest.mark.parametrize("types", xent_sizes.TYPES)
def test_ordinary_tokens(q8, T, V, K, types):  # noqa: F811
    """The other tests' rows with miss: their bounds hold, and tokens that do not count or are not
    finite are what they are without it."""
    c = Case(T, V, K)
    miss = torch.empty(T, device="cuda")
    loss, lse = c.forward(q8, miss=miss)
    c.check_forward(loss, lse)
    c.check_backward(*c.backward(q8, lse, *types, miss=miss), *types)
    c.target[T // 2], c.g[T // 2] = V, 1.0
    loss, lse = c.forward(q8, miss=miss)
    dx, dw = c.backward(q8, lse, *types, miss=miss)
    assert bool(dx[T // 2].isnan().all()) and bool(dw.isnan().all())


@pytest.mark.parametrize("T,V", [(9, 700), (40, 700), (300, 700)])
def test_captured(q8, T, V):  # noqa: F811
    c, miss = Confident(T, V, 100), torch.empty(T, device="cuda")
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    out = [torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda"),
           torch.zeros((T, 48), device="cuda")[:, :40], torch.zeros((V, 48), device="cuda")[:, :40]]

    def step():
        q8.cpdp_q8_xent(*c.held(), *out[:2], workspace=ws, miss=miss)
        q8.cpdp_q8_xent_bwd(*c.held(), out[1], c.g, *out[2:], workspace=ws, miss=miss)

    step()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        step()
    for shift in (1, 2, 3):
        c.target.copy_(c.target.roll(shift))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (*out, miss)]
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, (*out, miss)))


def test_refusals(q8):  # noqa: F811
    c = Confident(6, 40, 0)
    loss, lse = c.forward(q8)
    for bad, what in ((loss[:5], "vector"), (loss.double(), "float32"), (loss.cpu(), "GPU"),
                      (torch.empty(12, device="cuda")[::2], "vector")):
        with pytest.raises(ValueError, match=what):
            c.forward(q8, miss=bad)
        with pytest.raises(ValueError, match=what):
            c.backward(q8, lse, 0, 0, miss=bad)


def test_a_head_s_gradients_are_those_of_its_miss(q8):  # noqa: F811
    """Whatever the caller does with the losses that it was given."""
    from paper_2607_21224_amd.layer import Q8Head
    T, D, V = 96, 64, 300
    head, g = Q8Head(D, V, act_dt="f32"), torch.Generator(device="cuda").manual_seed(1)
    row = head.init(g)
    target = torch.randint(0, V, (T,), generator=g, device="cuda")
    x = torch.randn((T, D), generator=g, device="cuda") + 60 * head.view(row, "w")[target]
    head.view(row, "norm").fill_(8.0)  # steep: most tokens are confident
    s, grads = head.saved(T), torch.zeros(head.numel, device="cuda")
    weight = torch.rand(T, generator=g, device="cuda")
    loss = head.forward(row, x, target, s)
    assert float(loss.median()) < 1e-3
    miss, dx = torch.empty(T, device="cuda"), torch.empty((T, D), device="cuda")
    dw = torch.empty((V, D), device="cuda")
    q8.cpdp_q8_xent(s.n, s.n_scale, *s.w, target, loss.clone(), s.lse, miss=miss)
    q8.cpdp_q8_xent_bwd(s.n, s.n_scale, *s.w, target, s.lse, weight, dx, dw, miss=miss)
    loss.zero_()
    head.backward(row, weight, s, grads)
    assert torch.equal(s.dn, dx) and torch.equal(head.view(grads, "w"), dw)


@pytest.mark.parametrize("T", [3, 40, 130])
def test_the_smallest_and_largest_targets(q8, T):  # noqa: F811
    """A token of the smallest target does not count, as any negative one; one of the largest has
    no class."""
    c, ref = Confident(T, 700, 50), Confident(T, 700, 50)
    miss = torch.empty(T, device="cuda")
    c.target[1], ref.target[1] = -2 ** 63, -1
    for types in xent_sizes.TYPES:
        out = []
        for v in (c, ref):
            loss, lse = v.forward(q8, miss=miss)
            out.append((loss, lse, miss.clone(), *v.backward(q8, lse, *types, miss=miss)))
        assert all(torch.equal(a, b) for a, b in zip(*out)) and float(out[0][0][1]) == 0
    c.target[1] = 2 ** 63 - 1
    loss, lse = c.forward(q8, miss=miss)
    dx, dw = c.backward(q8, lse, 0, 0, miss=miss)
    assert bool(loss[1].isnan() & miss[1].isnan() & dx[1].isnan().all() & dw.isnan().all())
    others = torch.arange(T, device="cuda") != 1
    assert torch.equal(loss[others], out[0][0][others])
