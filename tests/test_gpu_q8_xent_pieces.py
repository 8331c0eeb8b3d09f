"""The loss' gradients in pieces of the classes that the laid-out weights bound, with the bounds
of test_gpu_q8_xent.py."""
import pytest
import torch

import xent_sizes
from test_gpu_q8 import q8  # noqa: F401
from test_gpu_q8_xent import DTYPE, Case
from xent_sizes import BF16

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("types", xent_sizes.TYPES + xent_sizes.ALONE)
@pytest.mark.parametrize("T,V,K", xent_sizes.WEIGHTS)
def test_gradients(q8, T, V, K, types):  # noqa: F811
    # (several pieces: one of all classes would need more than there is)
    dts = [DTYPE[max(t, 0)] for t in types]
    px = 1 if T <= 64 or types[0] == BF16 else 2
    room = q8.cpdp_q8_xent_bwd_workspace(T, V, K, *dts)
    if px == 2 or T <= 64:
        assert room < 2 * px * V * K
    c = Case(T, V, K)
    loss, lse = c.forward(q8)
    c.check_forward(loss, lse)
    got = c.backward(q8, lse, *types)
    c.check_backward(*got, *types)
    for a, b in zip(got, c.backward(q8, lse, *types)):
        assert a is None or torch.equal(a, b)


@pytest.mark.parametrize("T,V,K", xent_sizes.WEIGHTS[:3])
def test_captured(q8, T, V, K):  # noqa: F811
    c = Case(T, V, K)
    lse = c.forward(q8)[1]
    want = c.backward(q8, lse, 0, 1)
    ws = torch.empty(q8.cpdp_q8_xent_bwd_workspace(T, V, K, *DTYPE), dtype=torch.uint8,
                     device="cuda")
    dx, dw = (torch.empty_strided(v.shape, v.stride(), dtype=v.dtype, device="cuda") for v in want)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        q8.cpdp_q8_xent_bwd(*c.held(), lse, c.g, dx, dw, workspace=ws)
    for _ in range(3):
        dx.fill_(3), dw.fill_(3), ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])
