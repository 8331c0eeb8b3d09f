"""The MLP layer on the 8-bit path: its passes against float64 with the same 8-bit
operands, against autograd without rounding, and a training run whose steps are
the CPDP steps."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def held(q, s):
    return q.double() * s.double()[:, None]


def rel(x, y):
    return float((x.double() - y.double()).norm() / y.double().norm())


def act(kind, g, u):
    if kind == "gelu":
        return g * 0.5 * torch.erfc(-g / math.sqrt(2.0))
    return g * torch.sigmoid(g) * u


# one rounding to bfloat16 is at most 2^-8 of a value, 2^-8 / sqrt(3) in the 2-norm
B = 2.0 ** -8


@pytest.mark.parametrize("kind,act_dt,T,D,F", [("gelu", "bf16", 197, 384, 1536),
                                               ("swiglu", "bf16", 70, 128, 256),
                                               ("gelu", "f32", 33, 64, 200),
                                               ("swiglu", "f32", 500, 256, 512)])
def test_layer_against_float64(kind, act_dt, T, D, F):
    from paper_2607_21224_amd.layer import Q8Mlp
    mlp = Q8Mlp(D, F, kind, act_dt=act_dt)
    g, dt = gen(T), {"f32": torch.float32, "bf16": torch.bfloat16}[act_dt]
    row, grads = mlp.init(g), torch.zeros(mlp.numel, device="cuda")
    mlp.view(row, "norm").add_(0.1 * torch.randn(D, generator=g, device="cuda"))
    x, r, dy, dres = (torch.randn((T, D), generator=g, device="cuda").to(dt) for _ in range(4))
    s = mlp.saved(T)
    y = mlp.forward(row, x, s, residual=r)
    # the step after a rounding to 8 bits, from the 8-bit operands the layer used;
    # z is bf16 or fp32, then y
    one = B / math.sqrt(3.0) if act_dt == "bf16" else 1e-6
    z = [held(s.n, s.n_scale) @ held(*w).t().contiguous() for w in s.w1]
    assert all(rel(a, b) <= one for a, b in zip(s.z, z))
    assert rel(y, held(s.a, s.a_scale) @ held(*s.w2).t().contiguous()) <= one

    dx = mlp.backward(row, dy, s, grads, dres=dres).clone()
    # the same in float64 by autograd, roundings to 8 bits passed on unchanged
    d64 = lambda t: t.double().detach().requires_grad_(True)  # noqa: E731
    h, w0 = d64(s.h), d64(mlp.view(row, "norm"))
    n = h * (h.square().mean(1, keepdim=True) + mlp.eps).rsqrt() * w0
    w1 = [d64(held(*w)) for w in s.w1]
    w2 = d64(held(*s.w2))

    def through(v, value):
        return v + (value - v).detach()

    n8 = through(n, held(s.n, s.n_scale))
    G = through(n8 @ w1[0].t(), held(s.cg, s.g_scale))
    U = through(n8 @ w1[1].t(), held(s.cu, s.u_scale)) if mlp.gated else None
    a8 = through(act(kind, G, U), held(s.a, s.a_scale))
    ((a8 @ w2.t()) * dy.double()).sum().backward()
    # da, dz, dn and the results are rounded, and one operand of each product
    tol = 6 * B / math.sqrt(3.0) if act_dt == "bf16" else 1e-5
    assert rel(dx, h.grad + dres.double()) <= tol
    assert rel(mlp.view(grads, "norm"), w0.grad) <= tol
    assert rel(mlp.view(grads, "w1"), w1[0].grad) <= tol
    assert rel(mlp.view(grads, "w2"), w2.grad) <= tol
    if mlp.gated:
        assert rel(mlp.view(grads, "w1u"), w1[1].grad) <= tol


def test_training_with_the_cpdp_steps():
    """Four replicas learn a function of their inputs, each from its own batches, in
    periods of three steps: the loss falls as it does in float64 without any
    rounding, and after a synchronisation all replicas are the reference model."""
    from paper_2607_21224_amd.layer import Q8Mlp
    from paper_2607_21224_amd.state import CpdpState, Hyper
    W, K, D, F, T, steps = 4, 3, 64, 128, 96, 36
    mlp = Q8Mlp(D, F, "gelu", act_dt="f32")
    g = gen(1)
    theta = mlp.init(g)
    goal = torch.randn((D, D), generator=g, device="cuda") * D ** -0.5
    xs = torch.randn((W, T, D), generator=g, device="cuda")
    want = torch.tanh(xs @ goal)
    st = CpdpState(W=W, P=mlp.numel, K=K)
    st.init(theta)
    h = Hyper.fp32(lr=0.05, mu=0.9, beta=0.3, alpha=1.0)
    grads = torch.zeros((W, st.ld), device="cuda")
    s = mlp.saved(T)
    losses = []
    for t in range(1, steps + 1):
        loss = 0.0
        for i in range(W):
            err = mlp.forward(st.params[i], xs[i], s) - want[i]
            loss += float(err.square().sum(1).mean()) / W
            mlp.backward(st.params[i], err * (2.0 / T), s, grads[i])
        losses.append(loss)
        st.step(t, grads, h, steps)
        if t % K == 0:
            assert st.count_unsynced() == 0

    # the same run in float64, its gradients by autograd
    p = theta.double().repeat(W, 1)
    m, u, anchor = torch.zeros_like(p), torch.zeros_like(p[0]), theta.double()
    ref = []
    for t in range(1, steps + 1):
        gs, loss = [], 0.0
        for i in range(W):
            q = p[i].detach().requires_grad_(True)
            n = xs[i].double()
            n = n * (n.square().mean(1, keepdim=True) + mlp.eps).rsqrt() * mlp.view(q, "norm")
            a = act("gelu", n @ mlp.view(q, "w1").t(), None)
            out = a @ mlp.view(q, "w2").t() - want[i].double()
            one = out.square().sum(1).mean()
            loss += float(one.detach()) / W
            gs.append(torch.autograd.grad(one, q)[0])
        ref.append(loss)
        gs = torch.stack(gs)
        if t % K == 0:
            gs = gs.mean(0, keepdim=True).expand_as(p)
        m = 0.9 * m + gs
        p = p - 0.05 * m
        if t % K == 0:
            u = 0.3 * u + (anchor - p.mean(0)) / 0.05
            anchor = anchor - 0.05 * u
            p = anchor.repeat(W, 1)
    assert losses[-1] < 0.5 * losses[0]
    # 8 bits leave an error of up to 1 / 254 of a row's largest value in every
    # operand; the losses follow each other within a few per cent of the first
    assert all(abs(a - b) <= 0.03 * ref[0] for a, b in zip(losses, ref))


def test_layer_refusals():
    from paper_2607_21224_amd.layer import Q8Mlp
    with pytest.raises(ValueError, match="kind"):
        Q8Mlp(64, 64, "relu")
    with pytest.raises(ValueError, match="act_dt"):
        Q8Mlp(64, 64, act_dt="f16")
    with pytest.raises(ValueError, match="multiples of 8"):
        Q8Mlp(63, 64)
    mlp = Q8Mlp(64, 64)
    row, s = mlp.init(), mlp.saved(4)
    with pytest.raises(ValueError, match="q"):
        mlp.forward(row, torch.zeros((5, 64), dtype=torch.bfloat16, device="cuda"), s)
