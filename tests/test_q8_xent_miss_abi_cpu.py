"""What the calls of the loss with a token's miss refuse: all that those without it do, and a
miss that is not there, not aligned, past the address space or on another argument."""
import pytest
import torch

from paper_2607_21224_amd import q8
from test_q8_abi_cpu import DTYPE, INVALID, MISALIGNED, NULL, OK, OVERLAP, TOO_LARGE, at
from test_q8_xent_abi_cpu import CALLS as WITHOUT

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                reason="fake device addresses: CPU-only module")


def with_miss(args):
    out = {}
    for k, v in args.items():
        out[k] = v
        if k == "lse":
            out["miss"] = at(11)
    return out


CALLS = {"cpdp_q8_xent_miss": with_miss(WITHOUT["cpdp_q8_xent"]),
         "cpdp_q8_xent_miss_bwd": with_miss(WITHOUT["cpdp_q8_xent_bwd"])}


def call(name, **change):
    args = dict(CALLS[name])
    assert set(change) <= set(args)
    args.update(change)
    return getattr(q8.lib, name)(*args.values())


@pytest.mark.parametrize("name", CALLS)
def test_miss(name):
    a = CALLS[name]
    assert call(name, miss=None) == NULL
    assert call(name, miss=a["miss"] + 2) == MISALIGNED
    assert call(name, miss=(1 << 64) - 16) == INVALID
    written = ("dx", "dw") if "bwd" in name else [k for k, v in a.items() if k != "miss" and
                                                  isinstance(v, int) and v >= 1 << 40 and
                                                  k != "workspace"]
    for other in written:
        assert call(name, miss=a[other] + 16) == OVERLAP, other


@pytest.mark.parametrize("name", CALLS)
def test_the_others(name):
    assert call(name, T=-1) == call(name, V=0) == call(name, K=131072) == INVALID
    assert call(name, ldx=1 << 23) == TOO_LARGE
    pointers = [k for k, v in CALLS[name].items() if isinstance(v, int) and v >= 1 << 40]
    for k in pointers:
        if k not in ("dx", "dw", "workspace"):
            assert call(name, **{k: None}) == NULL, k
    if "bwd" in name:
        assert call(name, dx=None, dw=None) == NULL
        assert call(name, dx_dt=2) == call(name, dw_dt=-1) == DTYPE
        assert call(name, workspace_bytes=0) == INVALID
    gone = {k: None for k in pointers}
    assert call(name, **gone, T=0, workspace_bytes=0) == OK
