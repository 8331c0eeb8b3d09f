"""Q8Head on the streams a caller may name: the same bits on the current stream, the null
stream by its number, another by its handle and by its object."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def passes(head, T, stream):
    """Two passes over the same tensors, the second one's results."""
    g = torch.Generator(device="cuda").manual_seed(5)
    row, grads = head.init(g), torch.zeros(head.numel, device="cuda")
    x, r, dres = (torch.randn((T, head.dim), generator=g, device="cuda").to(head.act_dtype)
                  for _ in range(3))
    target = torch.randint(-1, head.classes, (T,), generator=g, device="cuda")
    weight = torch.rand(T, generator=g, device="cuda")
    s = head.saved(T)
    torch.cuda.synchronize()
    for _ in range(2):
        head.forward(row, x, target, s, residual=r, stream=stream)
        head.backward(row, weight, s, grads, dres=dres, stream=stream)
    torch.cuda.synchronize()
    return [t.clone() for t in (s.loss, s.lse, s.dx, grads)]


@pytest.mark.parametrize("act_dt,T,D,V", [("bf16", 300, 384, 5003), ("f32", 1, 64, 136),
                                          ("f32", 40, 128, 9001), ("bf16", 70, 64, 200)])
def test_streams(act_dt, T, D, V):
    from paper_2607_21224_amd.layer import Q8Head
    head = Q8Head(D, V, act_dt=act_dt)
    want = passes(head, T, None)
    assert all(bool(t.isfinite().all()) for t in want)
    side = torch.cuda.Stream()
    for stream in (0, side.cuda_stream, side):
        for a, b in zip(passes(head, T, stream), want):
            assert torch.equal(a, b), stream
