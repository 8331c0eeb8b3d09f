"""What a Q8Head refuses and keeps, on the CPU."""
import pytest
import torch

from paper_2607_21224_amd.layer import Q8Head
from test_q8_layer_memory_cpu import storages


def test_refusals():
    with pytest.raises(ValueError, match="act_dt"):
        Q8Head(64, 100, act_dt="f16")
    with pytest.raises(ValueError, match="multiple of 8"):
        Q8Head(63, 100)
    head = Q8Head(64, 100)
    row, s = head.init(device="cpu"), head.saved(4, device="cpu")
    x, target = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="GPU"):
        head.forward(row, x, target, s)


def test_layout():
    head = Q8Head(24, 11)
    row = head.init(device="cpu")
    assert row.shape == (head.numel,) and head.numel == 24 + 11 * 24
    assert bool((head.view(row, "norm") == 1).all())
    assert head.view(row, "w").shape == (11, 24) and bool((head.view(row, "w") != 0).all())
    head.view(row, "w")[3] = 7
    assert bool((row[24 + 3 * 24:24 + 4 * 24] == 7).all())


@pytest.mark.parametrize("act_dt,e", [("bf16", 2), ("f32", 4)])
def test_no_logits_are_kept(act_dt, e):
    T, D, V = 8192, 1024, 131072
    head = Q8Head(D, V, act_dt=act_dt)
    s = head.saved(T, device="meta")
    own = {k: v for k, v in vars(s).items() if k != "workspace"}
    count = 0
    for v in own.values():
        for t in v if isinstance(v, tuple) else (v,):
            if isinstance(t, torch.Tensor):
                count += t.numel() * t.element_size()
    # n, its scales, rstd, loss and lse, h, dn and dx, the weights in 8 bits
    assert count == T * (D + 4 * 4 + 3 * e * D) + V * (D + 4)
    # a piece's logits' gradients, laid out, and not T x V fp32 numbers
    parts = 6 if act_dt == "f32" else 4
    assert head.workspace_bytes(T) < parts * 2 ** 28 + 4 * T * V // 4
    assert head.workspace_bytes(T) < 4 * T * V


def test_tensors_of_a_saved_pass_are_its_own():
    head = Q8Head(64, 100)
    a, b = head.saved(8, device="cpu"), head.saved(8, device="cpu")
    assert not set(storages(a)) & set(storages(b))
