"""A stack of Q8Mlp layers that share what passes need for a while has the bits of one in
which every layer has its own."""
import pytest
import torch

from test_gpu_q8_layer import gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,act_dt", [("gelu", "bf16"), ("swiglu", "bf16"), ("gelu", "f32")])
def test_a_stack(kind, act_dt):
    from paper_2607_21224_amd.layer import Q8Mlp
    T, D, F, L = 150, 128, 256, 3
    mlp = Q8Mlp(D, F, kind, act_dt=act_dt)
    g = gen(7)
    rows = [mlp.init(g) for _ in range(L)]
    x, r0, dy = (torch.randn((T, D), generator=g, device="cuda").to(mlp.act_dtype)
                 for _ in range(3))
    results = []
    for shared in (False, True):
        scratch = mlp.scratch(T) if shared else None
        saved = [mlp.saved(T, scratch=scratch) for _ in range(L)]
        grads = [torch.zeros(mlp.numel, device="cuda") for _ in range(L)]
        for replica in range(2):  # one after the other over the same tensors
            y, r = x, r0
            for row, s in zip(rows, saved):
                y = mlp.forward(row, y, s, residual=r)
                r = s.h
            d, dres = dy, None
            for row, s, gr in zip(rows[::-1], saved[::-1], grads[::-1]):
                d = mlp.backward(row, d, s, gr, dres=dres)
                dres = d
        results.append([t.clone() for s in saved for t in (s.h, s.y, s.dx)] + grads)
    for a, b in zip(*results):
        assert torch.equal(a, b)
        assert bool(torch.isfinite(a).all()) and float(a.float().abs().max()) > 0
