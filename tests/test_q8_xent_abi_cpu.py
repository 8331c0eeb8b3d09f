"""What the loss refuses, on the host before any GPU work: only calls that fail validation or
have nothing to do are made, with fake aligned addresses that are never read."""
import pytest
import torch

from paper_2607_21224_amd import cpdp, q8
from test_q8_abi_cpu import (BF16, DTYPE, F32, INVALID, MISALIGNED, NULL, OK, OVERLAP, TOO_LARGE,
                             at)

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                reason="fake device addresses: CPU-only module")

CALLS = {
    "cpdp_q8_xent": dict(x=at(0), ldx=64, x_scale=at(1), w=at(2), ldw=64, w_scale=at(3),
                         target=at(4), T=80, V=32, K=64, loss=at(5), lse=at(6), workspace=at(7),
                         workspace_bytes=1 << 30, stream=None),
    "cpdp_q8_xent_bwd": dict(x=at(0), ldx=64, x_scale=at(1), w=at(2), ldw=64, w_scale=at(3),
                             target=at(4), lse=at(5), g=at(6), T=80, V=32, K=64, dx=at(7),
                             lddx=64, dx_dt=BF16, dw=at(8), lddw=64, dw_dt=F32, workspace=at(9),
                             workspace_bytes=1 << 30, stream=None),
}
POINTERS = [(n, k) for n, a in CALLS.items() for k, v in a.items()
            if isinstance(v, int) and v >= 1 << 40]
WRITTEN = {"cpdp_q8_xent": "loss lse workspace", "cpdp_q8_xent_bwd": "dx dw workspace"}


def call(name, **change):
    args = dict(CALLS[name])
    assert set(change) <= set(args)
    args.update(change)
    return getattr(q8.lib, name)(*args.values())


def workspace(name, **change):
    a = {**CALLS[name], **change}
    sizes = ("T", "V", "K") + (("dx_dt", "dw_dt") if "bwd" in name else ())
    return getattr(q8.lib, name + "_workspace")(*[a[k] for k in sizes])


@pytest.mark.parametrize("name", CALLS)
def test_counts(name):
    for change in (dict(T=-1), dict(T=1 << 31), dict(T=q8.CPDP_Q8_MAX_T + 1), dict(V=0),
                   dict(V=-1), dict(V=1 << 31), dict(K=0), dict(K=-4), dict(K=65),
                   dict(K=131072, ldx=131072, ldw=131072, **(
                       dict(lddx=131072, lddw=131072) if "bwd" in name else {}))):
        assert call(name, **change) == INVALID, change
        if "K" not in change or change["K"] != 65:
            assert workspace(name, **change) == 0


@pytest.mark.parametrize("name,which", POINTERS)
def test_pointers(name, which):
    if which not in ("dx", "dw") and not (which == "workspace" and workspace(name) == 0):
        assert call(name, **{which: None}) == NULL
    step = 4 if which == "target" else 2 if which in ("x_scale", "w_scale", "loss", "lse",
                                                       "g") else 8
    if which != "workspace" or workspace(name) > 0:
        assert call(name, **{which: CALLS[name][which] + step}) == MISALIGNED
        assert call(name, **{which: (1 << 64) - 16}) == INVALID


def test_a_gradient_at_least():
    assert call("cpdp_q8_xent_bwd", dx=None, dw=None) == NULL


@pytest.mark.parametrize("name,which", [(n, k) for n, a in CALLS.items() for k in a
                                        if k.startswith("ld")])
def test_strides(name, which):
    assert call(name, **{which: 16}) == INVALID
    assert call(name, **{which: 68 + 1}) == MISALIGNED
    assert call(name, **{which: -64}) == INVALID
    assert call(name, **{which: 1 << 29}) == INVALID
    if which in ("ldx", "ldw"):
        assert call(name, **{which: 1 << 23}) == TOO_LARGE


@pytest.mark.parametrize("which", ["dx_dt", "dw_dt"])
def test_storage_types(which):
    for code in (2, -1):
        assert call("cpdp_q8_xent_bwd", **{which: code}) == DTYPE
        assert workspace("cpdp_q8_xent_bwd", **{which: code}) == 0


@pytest.mark.parametrize("name,out,other", [(n, o, k) for n in CALLS for o in WRITTEN[n].split()
                                            for m, k in POINTERS if m == n and o != k])
def test_overlaps(name, out, other):
    if "workspace" in (out, other) and workspace(name) < 64:
        return
    assert call(name, **{out: CALLS[name][other] + 16}) == OVERLAP


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("T,V,K", [(1, 32768, 64), (80, 32, 64), (300, 5000, 64), (5000, 300, 64),
                                   (2097088, 2, 1)])
def test_workspaces(name, T, V, K):
    sizes = dict(T=T, V=V, K=K)
    need = workspace(name, **sizes)
    assert need % 16 == 0
    if need > 0:
        assert call(name, **sizes, workspace_bytes=need - 1) == INVALID
        assert call(name, **sizes, workspace=None, workspace_bytes=need) == NULL
        last = at(0) + 16 - need
        assert call(name, **sizes, workspace=last, workspace_bytes=need) == OVERLAP


def test_no_tokens():
    gone = dict(x=None, x_scale=None, w=None, w_scale=None, target=None, T=0)
    assert call("cpdp_q8_xent", **gone, loss=None, lse=None, workspace=None,
                workspace_bytes=0) == OK
    assert call("cpdp_q8_xent_bwd", **gone, lse=None, g=None, dx=None, dw=None, workspace=None,
                workspace_bytes=0) == OK
    assert call("cpdp_q8_xent_bwd", **gone, lse=None, g=None, dw=None, workspace=None,
                workspace_bytes=0) == OK
    assert workspace("cpdp_q8_xent", T=0) == workspace("cpdp_q8_xent_bwd", T=0) == 0


def test_the_largest_number_of_tokens_is_that_of_the_header():
    text = open(f"{cpdp._PKG}/../include/cpdp_q8.h").read()
    assert f"#define CPDP_Q8_MAX_T {q8.CPDP_Q8_MAX_T} " in text


def test_python_checks_come_first():
    x, s = torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4)
    w, t = torch.zeros(9, 32, dtype=torch.int8), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="current GPU"):
        q8.cpdp_q8_xent(x, s, w, torch.zeros(9), t, s, s)
    with pytest.raises(ValueError, match="torch.int8|Char"):
        q8.cpdp_q8_xent(x.float(), s, w, torch.zeros(9), t, s, s)
