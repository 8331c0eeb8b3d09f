"""Errors of the 8-bit path's binding that need a GPU."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_no_memory_for_a_workspace():
    """A workspace that torch's allocator cannot give is torch's own error, and the
    call goes through once there is memory."""
    from paper_2607_21224_amd import q8
    T = N = K = 4096
    dy = torch.zeros(T, N, device="cuda")
    b, s = torch.ones(N, K, dtype=torch.int8, device="cuda"), torch.ones(N, device="cuda")
    dx = torch.ones(T, K, device="cuda")
    need = q8.cpdp_q8_grad_input_workspace(T, N, K, dy.dtype, dx.dtype)
    assert need > 64 << 20
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    total = torch.cuda.get_device_properties(0).total_memory
    held = []
    try:
        torch.cuda.set_per_process_memory_fraction(
            (torch.cuda.memory_reserved() + (8 << 20)) / total)
        # what the allocator has kept of earlier tests
        with pytest.raises(torch.OutOfMemoryError):
            while True:
                held.append(torch.empty(48 << 20, dtype=torch.uint8, device="cuda"))
        with pytest.raises(torch.OutOfMemoryError):
            q8.cpdp_q8_grad_input(dy, b, s, dx)
    finally:
        held.clear()
        torch.cuda.set_per_process_memory_fraction(1.0)
    assert bool((dx == 1).all())
    q8.cpdp_q8_grad_input(dy, b, s, dx)
    assert bool((dx == 0).all())
