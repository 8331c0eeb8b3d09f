"""Q8Mlp on the streams a caller may name: the same bits on the current stream, the null
stream by its number, another by its handle and by its object; and the gated kind's sum
over both halves against float64."""
import math

import pytest
import torch

from test_gpu_q8_layer import B, gen, held, rel

pytestmark = pytest.mark.gpu


def passes(mlp, T, stream):
    """Two passes over the same tensors, the second one's results."""
    g = gen(5)
    row, grads = mlp.init(g), torch.zeros(mlp.numel, device="cuda")
    x, r, dy = (torch.randn((T, mlp.dim), generator=g, device="cuda").to(mlp.act_dtype)
                for _ in range(3))
    s = mlp.saved(T)
    torch.cuda.synchronize()
    for _ in range(2):
        mlp.forward(row, x, s, residual=r, stream=stream)
        mlp.backward(row, dy, s, grads, stream=stream)
    torch.cuda.synchronize()
    return [t.clone() for t in (s.y, s.dx, grads)]


@pytest.mark.parametrize("kind,act_dt,T,D,F", [("swiglu", "bf16", 300, 384, 512),
                                               ("swiglu", "f32", 1, 64, 136),
                                               ("gelu", "bf16", 300, 384, 512)])
def test_streams(kind, act_dt, T, D, F):
    from paper_2607_21224_amd.layer import Q8Mlp
    mlp = Q8Mlp(D, F, kind, act_dt=act_dt)
    want = passes(mlp, T, None)
    side = torch.cuda.Stream()
    for stream in (0, side.cuda_stream, side):
        for a, b in zip(passes(mlp, T, stream), want):
            assert torch.equal(a, b), stream


@pytest.mark.parametrize("act_dt,T,D,F", [("bf16", 200, 256, 512), ("f32", 70, 64, 200),
                                          ("f32", 1, 64, 40)])
def test_the_gated_kind_s_gradient_of_the_norm_s_output(act_dt, T, D, F):
    """One sum over the channels of both halves.  bf16: one operand and the result are
    rounded, each up to 2^-8 / sqrt(3) of the 2-norm; fp32 sums err by 2e-6 or less of it."""
    from paper_2607_21224_amd.layer import Q8Mlp
    mlp = Q8Mlp(D, F, "swiglu", act_dt=act_dt)
    g = gen(T)
    row, grads = mlp.init(g), torch.zeros(mlp.numel, device="cuda")
    x, dy = (torch.randn((T, D), generator=g, device="cuda").to(mlp.act_dtype) for _ in range(2))
    s = mlp.saved(T)
    mlp.forward(row, x, s)
    mlp.backward(row, dy, s, grads)
    # (s.z holds the gradient of z after the backward pass)
    want = sum(dz.double() @ held(*w) for dz, w in zip(s.z, s.w1))
    assert rel(s.dn, want) <= (math.sqrt(2.0 / 3.0) * B if act_dt == "bf16" else 2e-6)
    for name, dz in zip(("w1", "w1u"), s.z):
        want = dz.double().t() @ held(s.n, s.n_scale)
        tol = math.sqrt(2.0 / 3.0) * B if act_dt == "bf16" else 2e-6
        assert rel(mlp.view(grads, name), want) <= tol
