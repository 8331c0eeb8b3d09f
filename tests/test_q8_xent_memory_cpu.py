"""The workspace of the loss' gradients: bounded whatever the number of classes, and what a
Q8Head allocates with few tokens over a large vocabulary."""
import itertools

import pytest
import torch

from paper_2607_21224_amd import q8
from paper_2607_21224_amd.layer import Q8Head
from test_q8_abi_cpu import BF16, F32

MIB = 1 << 20
TYPES = list(itertools.product((F32, BF16), repeat=2))


def most(T, K):
    """The bound that cpdp_q8.h gives."""
    rows = 12 * (T + 64) * (K + 64)
    return 512 * MIB if T <= 64 else max(1024 * MIB, 2048 * T) + 640 * MIB + rows


@pytest.mark.parametrize("T", [1, 16, 17, 32, 33, 40, 64, 65, 70, 128, 200, 1024, 2049, 8192, 30000,
                               1 << 18, q8.CPDP_Q8_MAX_T])
def test_bounded_whatever_the_classes(T):
    for V, K, types in itertools.product((1, 100, 32768, 151936, 1000000, 20000003, (1 << 31) - 9),
                                         (1, 100, 1024, 4096, 20000, 131071), TYPES):
        need = q8.lib.cpdp_q8_xent_bwd_workspace(T, V, K, *types)
        assert 0 < need <= most(T, K), (V, K, types, need // MIB, most(T, K) // MIB)


@pytest.mark.parametrize("T,mib", [(1, 32), (32, 32), (33, 160), (64, 160), (65, 560), (128, 560),
                                   (1024, 900)])
def test_few_tokens_over_a_large_vocabulary(T, mib):
    """151936 classes of 4096 channels: 622 MB in 8 bits, 1244 in fp16 numbers."""
    assert Q8Head(4096, 151936).workspace_bytes(T) <= mib * MIB


def test_meta_allocation():
    """What a pass of 128 tokens allocates in all, beside the weights in 8 bits."""
    s = Q8Head(4096, 151936).saved(128, device="meta")
    total = 0
    for v in vars(s).values():
        for t in v if isinstance(v, tuple) else (v,):
            if isinstance(t, torch.Tensor):
                total += t.numel() * t.element_size()
    assert total - 151936 * (4096 + 4) <= 600 * MIB
