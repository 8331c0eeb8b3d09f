"""Workspaces of the 8-bit path on the CPU, with sizes that need one: a smaller one, none, one
off its boundary and one that overlaps an argument are refused before any GPU work.  Only
refused calls are made, with fake addresses."""
import pytest
import torch

from paper_2607_21224_amd import q8
from test_q8_abi_cpu import (BF16, CALLS, F32, INVALID, MISALIGNED, NULL, OVERLAP, POINTERS,
                             call)

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                reason="fake device addresses: CPU-only module")

# what of each call is changed so that its kernels need room
SIZES = [
    ("cpdp_q8_norm_bwd", dict(T=5000, D=64), ("T", "D")),
    ("cpdp_q8_norm_bwd", dict(T=9, D=40000, lddy=40000, ldh=40000, lddres=40000, lddx=40000),
     ("T", "D")),
    # a product whose sum is cut into slices
    ("cpdp_q8_matmul", dict(M=100, N=304, K=4096, lda=4096, ldb=4096, ldy=304), ("M", "N", "K")),
    # laid out; fp32 gradients with the 8-bit operand laid out; few tokens in slices
    ("cpdp_q8_grad_input", dict(T=200), ("T", "N", "K", "dy_dt", "out_dt")),
    ("cpdp_q8_grad_input", dict(T=1576, N=1536, lddy=1536, K=384, ldb=384, lddx=384, dy_dt=F32),
     ("T", "N", "K", "dy_dt", "out_dt")),
    ("cpdp_q8_grad_input", dict(T=5, N=320, lddy=320), ("T", "N", "K", "dy_dt", "out_dt")),
    ("cpdp_q8_grad_weight", dict(T=1025, out_dt=BF16), ("T", "N", "K", "dy_dt", "out_dt")),
]


@pytest.mark.parametrize("name,change,sizes", SIZES)
def test_a_workspace_that_does_not_do(name, change, sizes):
    args = {**CALLS[name], **change}
    need = getattr(q8.lib, name + "_workspace")(*[args[k] for k in sizes])
    assert need > 0 and need % 16 == 0
    base = dict(change, workspace_bytes=need)
    assert call(name, **{**base, "workspace_bytes": need - 1}) == INVALID
    assert call(name, **{**base, "workspace_bytes": 0}) == INVALID
    assert call(name, **base, workspace=None) == NULL
    assert call(name, **base, workspace=args["workspace"] + 8) == MISALIGNED
    for other in POINTERS[name]:
        if other != "workspace":
            # on its first bytes, and on the workspace's last ones
            assert call(name, **base, workspace=args[other]) == OVERLAP, other
            assert call(name, **base, workspace=args[other] + 16 - need // 16 * 16) == OVERLAP


def test_what_needs_none_takes_none():
    assert q8.lib.cpdp_q8_matmul_workspace(64, 304, 4096) == 0
    assert q8.lib.cpdp_q8_grad_weight_workspace(64, 304, 4096, F32, F32) == 0
    # a size that the call refuses
    assert q8.lib.cpdp_q8_matmul_workspace(100, 304, 131072) == 0
    assert q8.lib.cpdp_q8_matmul_workspace(-1, 304, 64) == 0
    assert q8.lib.cpdp_q8_norm_bwd_workspace(8, 0) == 0
    assert q8.lib.cpdp_q8_grad_input_workspace(200, 32, 64, 7, F32) == 0
