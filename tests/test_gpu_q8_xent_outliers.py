"""Gradients of the loss where one scale is far above the others: past 64 tokens they are held in
fp16 numbers over a common power of two, and what is lost is as much of the largest scale as the
header says.  The outlier's row is zero, so that nothing of it hides the others' error."""
import pytest
import torch

import xent_sizes
from test_gpu_q8 import q8  # noqa: F401
from test_gpu_q8_xent import Case

pytestmark = pytest.mark.gpu

SIZES = [(9, 700, 128), (65, 700, 128), (100, 70, 384), (700, 3001, 130), (2600, 4100, 64)]


@pytest.mark.parametrize("power", [10, 20, 40])
@pytest.mark.parametrize("which", ["class", "token", "weight"])
@pytest.mark.parametrize("types", xent_sizes.TYPES)
@pytest.mark.parametrize("T,V,K", SIZES)
def test_an_outlier(q8, T, V, K, types, which, power):  # noqa: F811
    c = Case(T, V, K, seed=power, ignored=0.0)
    t, v, most = T // 2, V // 3, 2.0 ** power
    if which == "class":
        c.w[v], c.ws[v] = 0, most * c.ws.max()
    elif which == "token":
        c.x[t], c.xs[t] = 0, most * c.xs.max()
    else:
        c.g[t] = most * c.g.abs().max()
    loss, lse = c.forward(q8)
    c.check_forward(loss, lse)
    c.check_backward(*c.backward(q8, lse, *types), *types)


@pytest.mark.parametrize("T", [65, 300])
def test_a_token_that_does_not_count_takes_no_bits(q8, T):  # noqa: F811
    """Its scale and weight are not among those that the power of two is found from: the others'
    gradients keep their bits whatever they are."""
    a, b = (Case(T, 700, 128, ignored=0.0) for _ in range(2))
    for c in (a, b):
        c.target[5] = -1
    b.xs[5], b.g[5] = 2.0 ** 60, 2.0 ** 50
    for types in xent_sizes.TYPES:
        x = a.backward(q8, a.forward(q8)[1], *types)
        y = b.backward(q8, b.forward(q8)[1], *types)
        assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])
