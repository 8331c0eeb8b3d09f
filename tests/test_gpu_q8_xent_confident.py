"""The loss of tokens whose target has nearly all of the probability, at large logits that
fp32 holds exactly: what is lost there is the loss' own.

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
"""
import math

import pytest
import torch

from test_gpu_q8 import U, q8  # noqa: F401

pytestmark = pytest.mark.gpu

GAP = 5.75  # and twice and three times that
SIZES = [(1, 33), (9, 700), (16, 5003), (40, 5003), (65, 700), (130, 33), (300, 5003)]


class Confident:
    def __init__(self, T, V, base, K=40, pad=0):
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

    def held(self):
        return self.x, self.xs, self.w, self.ws, self.target

    def forward(self, q8, **kw):  # noqa: F811
        loss, lse = (torch.empty(self.T, device="cuda") for _ in range(2))
        q8.cpdp_q8_xent(*self.held(), loss, lse, **kw)
        return loss, lse


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
