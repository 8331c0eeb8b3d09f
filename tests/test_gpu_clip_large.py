"""Clipping of gradients past 64 MB, which are scaled by blocks of their own, each by its row's
norm or the mean's, against 64 bits with the bounds of test_gpu_clip.py: rows that are scaled
beside rows that are not, and a norm that no row is scaled by."""
import math

import pytest
import torch

from paper_2607_21224_amd.multi import CpdpMultiState
from test_gpu_clip import bits, check_flat, clipped64, fill, norms64

pytestmark = pytest.mark.gpu

# (all past 67,108,864 bytes)
SIZES = [(5, (1 << 22) + 13, "f32"), (2, (1 << 23) + 1, "f32"), (9, (1 << 22) + 13, "bf16"),
         (1, (1 << 25) + 7, "bf16"), (300, 60001, "f32")]


@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("W,P,dt", SIZES)
def test_flat_rows(W, P, dt, mean):
    assert W * P * (4 if dt == "f32" else 2) > 64 << 20
    # the rows' norms are sqrt(P) e^-2 to sqrt(P) e^2, the mean's sqrt(P) / W times their length
    for share in (0.1, 1.0, 100.0):
        check_flat(W, P, dt, mean, max_norm=share * math.sqrt(P), seed=W)


@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("W", [1, 3, 5])
def test_tensors(W, mean):
    """(their rows' lengths are sqrt(P) times 1, 1.4, 1.9 ..)"""
    numels = [(1 << 24) // W + 7, 1, 0, 4096, (1 << 20) + 3, 17]
    P = sum(numels)
    assert 4 * W * P > 64 << 20
    st = CpdpMultiState(W, numels)
    fill(st, W)
    before = torch.stack([st.gather("grads", i) for i in range(W)])
    want, off = norms64(before, P, mean)
    for share in (100.0, 1.6, 0.3):
        max_norm = share * math.sqrt(P)
        norm = st.clip_grads(max_norm, mean)
        assert ((norm.double() - want).abs() <= off).all()
        after = torch.stack([st.gather("grads", i) for i in range(W)])
        values, room, same = clipped64(before, P, norm.double(), max_norm, "f32")
        assert ((after.double() - values).abs() <= room).all()
        assert all(torch.equal(bits(after[i]), bits(before[i])) for i in range(W) if same[i])
        for row in st.grads:
            for x, n in zip(row, numels):
                assert x[n:].isnan().all()
        fill(st, W)
