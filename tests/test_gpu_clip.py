"""Gradient norms and clipping against 64 bits.

Bounds, with u = 2^-24 half a step of fp32:
  norm      squares and sums are fp64: what is off is its rounding to fp32, u
  mean      gbar is W fp32 sums and a product: off by (W + 1) u sum_i |g_i| / W at most for
            each coordinate, and a norm by no more than the norm of that
  scaled    norm, norm + 1e-6, the quotient and the product are rounded once each: 4 u, and
            half a step of bf16 (2^-8) where that is what is stored
"""
import math

import pytest
import torch

from paper_2607_21224_amd import cpdp
from paper_2607_21224_amd.multi import CpdpMultiState
from paper_2607_21224_amd.state import CpdpState, Hyper, Optimizer

pytestmark = pytest.mark.gpu

U = 2.0 ** -24 * (1 + 1e-6)
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(W, P, dt, seed=0, sigma=1.0, pad=None):
    """(W, ld) gradients with NaN between the rows' ends and the next rows' starts."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    ld = (P + 7) // 8 * 8 + (16 if pad is None else pad)
    g = torch.full((W, ld), float("nan"), dtype=DT[dt], device="cuda")
    size = sigma * torch.exp(torch.linspace(-2, 2, W, device="cuda"))[:, None]
    g[:, :P] = torch.randn((W, P), generator=gen, device="cuda") * size
    return g, ld


def norms64(g, P, mean):
    """The norms in 64 bits, and how far off they may be."""
    v = g[:, :P].double()
    if not mean:
        n = v.square().sum(1).sqrt()
        return n, n * U
    W = len(v)
    n = v.mean(0).square().sum().sqrt().reshape(1)
    off = ((W + 1) * U * v.abs().mean(0)).square().sum().sqrt()
    return n, n * U + off


def clipped64(g, P, norm, max_norm, dt):
    c = torch.minimum(max_norm / (norm + 1e-6), torch.ones_like(norm)).reshape(-1, 1)
    want = g[:, :P].double() * c
    rel = 4 * U + (2.0 ** -8 if dt == "bf16" else 0)
    return want, want.abs() * rel * (1 + 1e-3) + 2.0 ** -140, (c == 1).expand(len(g), 1)


def workspace(W, P):
    return torch.full((cpdp.cpdp_grad_norm_workspace(W, P),), 255, dtype=torch.uint8, device="cuda")


def bits(x):
    return x.view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32)


def check_flat(W, P, dt, mean, max_norm, seed=0, sigma=1.0):
    g, ld = make(W, P, dt, seed, sigma)
    before = g.clone()
    n = 1 if mean else W
    ws = workspace(W, P)
    flags = cpdp.CPDP_NORM_MEAN if mean else 0
    want, off = norms64(g, P, mean)
    norm = torch.full((n + 1,), -7.0, device="cuda")
    cpdp.cpdp_grad_norm(g, W, P, ld, norm[:n], ws, dt, flags)
    assert torch.equal(bits(g), bits(before))
    assert ((norm[:n].double() - want).abs() <= off).all() and norm[n] == -7
    again = torch.full((n + 1,), -7.0, device="cuda")
    cpdp.cpdp_clip_grads(g, W, P, ld, max_norm, again[:n], ws, dt, flags)
    assert again[n] == -7
    assert ((again[:n].double() - want).abs() <= off).all()
    # the scale comes from the norm that the call found
    values, room, same = clipped64(before, P, again[:n].double(), max_norm, dt)
    assert ((g[:, :P].double() - values).abs() <= room).all()
    for i in range(W):
        if same[i]:
            assert torch.equal(bits(g[i]), bits(before[i]))
    assert torch.equal(bits(g[:, P:].contiguous()), bits(before[:, P:].contiguous()))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("P", [1, 2, 3, 4, 7, 8, 9, 255, 256, 257, 1023, 1024, 1025, 4101, 8200,
                               100003, 1048589])
def test_flat_rows(P, mean, dt):
    for W in (1, 2, 3, 8, 13):
        check_flat(W, P, dt, mean, max_norm=math.sqrt(P) * (0.3 if mean else 1.0), seed=P + W)


@pytest.mark.parametrize("W,P", [(33, 5003), (100, 70001), (2049, 5), (3000, 300)])
@pytest.mark.parametrize("mean", [False, True])
def test_many_replicas(W, P, mean):
    check_flat(W, P, "f32", mean, max_norm=math.sqrt(P) * 0.2)
    check_flat(W, P, "bf16", mean, max_norm=math.sqrt(P) * 0.2)


def test_offsets_past_32_bits():
    P = (1 << 31) + 13
    g = torch.zeros((1, P + 3), dtype=torch.bfloat16, device="cuda")
    g[0, P - 1], g[0, 5], g[0, 1 << 31] = 3.0, 4.0, 12.0
    norm = torch.empty(1, device="cuda")
    cpdp.cpdp_clip_grads(g, 1, P, P + 3, 6.5, norm, workspace(1, P), "bf16")
    assert norm.item() == 13.0
    assert (g[0, P - 1].item(), g[0, 5].item(), g[0, 1 << 31].item()) == (1.5, 2.0, 6.0)
    assert g.count_nonzero().item() == 3


@pytest.mark.parametrize("mean", [False, True])
def test_no_coordinates(mean):
    g = torch.full((3, 8), 5.0, device="cuda")
    norm = torch.full((3,), -1.0, device="cuda")
    n = 1 if mean else 3
    cpdp.cpdp_clip_grads(g, 3, 0, 8, 1.0, norm, workspace(3, 0),
                         flags=cpdp.CPDP_NORM_MEAN if mean else 0)
    assert norm.tolist() == [0.0] * n + [-1.0] * (3 - n)
    assert (g == 5).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_small_and_large_values(dt):
    """Squares past fp32's range either way."""
    P = 5001
    for size in (1e-38, 1e-30, 1e30, 1e36):
        g = torch.zeros((2, 5008), dtype=DT[dt], device="cuda")
        g[:, :P] = size
        norm = torch.empty(2, device="cuda")
        want, off = norms64(g, P, False)
        cpdp.cpdp_grad_norm(g, 2, P, 5008, norm, workspace(2, P), dt)
        assert ((norm.double() - want).abs() <= off + 2.0 ** -149).all()


def test_zeros_infinities_and_nan():
    P = 3001
    g = torch.ones((5, 3008), device="cuda")
    g[0] = 0
    g[1, 77] = float("inf")
    g[2, 2999] = float("nan")
    g[3, :P] = 3e38  # a norm past fp32's range
    norm = torch.empty(5, device="cuda")
    cpdp.cpdp_clip_grads(g, 5, P, 3008, 2.0, norm, workspace(5, P))
    n = norm.tolist()
    assert n[0] == 0 and n[1] == n[3] == math.inf and math.isnan(n[2])
    assert (g[0] == 0).all()
    assert g[1, 77].isnan() and g[1, :P].count_nonzero() == 1 and g[1, 76] == 0
    assert g[2, :P].isnan().all() and (g[2, P:] == 1).all()
    assert (g[3, :P] == 0).all()
    assert abs(g[4, 0].item() - 2 / math.sqrt(P)) < 1e-6


NUMELS = [[1], [3], [256], [0, 5, 0, 257, 1], [64, 64, 64, 4096, 64, 7, 1000, 2048, 3],
          [9408, 64, 64, 4096, 64, 64, 36864, 1, 262144 + 3], [1] * 300, [0, 0, 2, 0],
          [100003, 5, 0, 524288, 17] * 3, [0]]


def fill(st, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    for i, row in enumerate(st.grads):
        for x, n in zip(row, st.numels):
            x.fill_(float("nan"))
            x[:n] = torch.randn(n, generator=gen, device="cuda") * math.exp(i / 3)


@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("W", [1, 4, 11])
@pytest.mark.parametrize("k", range(len(NUMELS)))
def test_tensors(k, W, mean):
    st = CpdpMultiState(W, NUMELS[k])
    fill(st, k)
    P = sum(NUMELS[k])
    before = torch.stack([st.gather("grads", i) for i in range(W)])
    max_norm = 0.4 * math.sqrt(max(P, 1))
    want, off = norms64(before, P, mean)
    assert ((st.grad_norm(mean).double() - want).abs() <= off).all()
    norm = st.clip_grads(max_norm, mean)
    assert norm.shape == (1 if mean else W,)
    assert ((norm.double() - want).abs() <= off).all()
    after = torch.stack([st.gather("grads", i) for i in range(W)])
    values, room, same = clipped64(before, P, norm.double(), max_norm, "f32")
    assert ((after.double() - values).abs() <= room).all()
    assert all(torch.equal(after[i], before[i]) for i in range(W) if same[i])
    for row in st.grads:
        for x, n in zip(row, st.numels):
            assert x[n:].isnan().all()


@pytest.mark.parametrize("mean", [False, True])
def test_same_bits_again(mean):
    g, ld = make(7, 300007, "f32", 3)
    out = []
    for _ in range(2):
        x, norm = g.clone(), torch.empty(1 if mean else 7, device="cuda")
        cpdp.cpdp_clip_grads(x, 7, 300007, ld, 1.0, norm, workspace(7, 300007),
                             flags=cpdp.CPDP_NORM_MEAN if mean else 0)
        out.append((bits(x), bits(norm)))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


@pytest.mark.parametrize("grad_dt", ["f32", "bf16"])
@pytest.mark.parametrize("method", ["cpdp", "localsgd", "ddp"])
def test_a_clipped_step(method, grad_dt):
    """clip_grads and step() as a training loop calls them, against steps on gradients that
    were clipped with the norms found."""
    W, P = 4, 5003
    h = Hyper.fp32(0.1, 0.9, 0.5, 1.0)
    a, b = (CpdpState(W, P, K=2, grad_dt=grad_dt) for _ in range(2))
    theta = torch.randn(P, device="cuda")
    a.init(theta), b.init(theta)
    for t in range(1, 5):
        g, _ = make(W, P, grad_dt, t, pad=a.ld - (P + 7) // 8 * 8)
        mean = method == "ddp" or (method == "cpdp" and t % 2 == 0)
        x = g.clone()
        norm = a.clip_grads(x, 20.0, mean)
        # (a quotient of two tensors: a number over one is a product with its reciprocal)
        scale = (torch.full_like(norm, 20.0) / (norm + 1e-6)).clamp(max=1.0).reshape(-1, 1)
        assert (scale < 1).any()
        y = (g.float() * scale).to(g.dtype)
        assert torch.equal(bits(x[:, :P].contiguous()), bits(y[:, :P].contiguous()))
        a.step(t, x, h, method=method), b.step(t, y, h, method=method)
    assert torch.equal(a.params[:, :P], b.params[:, :P])


def test_tensors_clipped_step():
    st = CpdpMultiState(2, [1000, 3, 70000], K=2)
    ref = CpdpMultiState(2, [1000, 3, 70000], K=2)
    th = [torch.randn(n, device="cuda") for n in st.numels]
    st.init(th), ref.init(th)
    opt = Optimizer("sgd", 0.1, 0.9)
    for t in (1, 2):
        fill(st, t), fill(ref, t)
        norm = st.clip_grads(5.0, mean=t == 2)
        scale = (torch.full_like(norm, 5.0) / (norm + 1e-6)).clamp(max=1.0).expand(2)
        for i in range(2):
            for x in ref.grads[i]:
                x.mul_(scale[i])
        st.step(t, opt), ref.step(t, opt)
    assert all(torch.equal(st.gather("params", i), ref.gather("params", i)) for i in range(2))


@pytest.mark.parametrize("mean", [False, True])
def test_captured(mean):
    """Two graphs of one state, replayed in turn with eager calls between."""
    st = CpdpState(3, 100001)
    gs = [make(3, 100001, "f32", s, pad=st.ld - 100008)[0] for s in (1, 2)]
    want = [(x, st.clip_grads(x, 50.0, mean)) for x in (g.clone() for g in gs)]
    bufs = [torch.empty_like(g) for g in gs]
    graphs, norms = [], []
    side = torch.cuda.Stream()
    for b in bufs:
        b.copy_(gs[0])
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            norms.append(st.clip_grads(b, 50.0, mean))
        graphs.append(graph)
    for _ in range(3):
        for k in (0, 1):
            bufs[k].copy_(gs[k])
            graphs[k].replay()
            assert torch.equal(bits(norms[k]), bits(want[k][1]))
            assert torch.equal(bits(bufs[k]), bits(want[k][0]))
            st.grad_norm(gs[1 - k], mean)
            torch.cuda.synchronize()


def test_on_a_stream():
    st = CpdpState(2, 40001)
    g = make(2, 40001, "f32", 5, pad=st.ld - 40008)[0]
    want = g.clone()
    st.clip_grads(want, 3.0)
    s, norm = torch.cuda.Stream(), torch.empty(2, device="cuda")
    torch.cuda.synchronize()
    for stream in (s, s.cuda_stream):
        x = g.clone()
        torch.cuda.synchronize()
        assert st.clip_grads(x, 3.0, norm=norm, stream=stream) is norm
        s.synchronize()
        assert torch.equal(bits(x), bits(want))
    with torch.cuda.stream(s):
        x = g.clone()
        st.clip_grads(x, 3.0)
    s.synchronize()
    assert torch.equal(bits(x), bits(want))
    with pytest.raises(ValueError, match="norm"):
        st.clip_grads(x, 3.0, stream=s)


@pytest.mark.parametrize("plan", [False, True])
def test_a_first_call_on_a_stream(plan):
    """It takes no memory: what torch's current stream still writes to stays out of it."""
    st = CpdpMultiState(2, [40001, 5]) if plan else CpdpState(2, 40001)
    of = () if plan else (torch.empty((2, st.ld), device="cuda"),)
    for t in sum(st.grads, []) if plan else of:
        t.fill_(1.0)
    s, norm = torch.cuda.Stream(), torch.empty(2, device="cuda")
    torch.cuda.synchronize()
    before = torch.cuda.memory_stats()["allocation.all.allocated"]
    st.grad_norm(*of, norm=norm, stream=s)
    st.clip_grads(*of, 3.0, norm=norm, stream=s)
    assert torch.cuda.memory_stats()["allocation.all.allocated"] == before
    s.synchronize()
    want = math.sqrt(40006 if plan else 40001)
    assert bool(((norm - want).abs() <= 2 * U * want).all())
