"""The C ABI of the 8-bit activation path on the CPU: it exports what its header
declares, and refuses wrong arguments on the host before any GPU work.  Only
calls that fail validation or have nothing to do are made, with fake aligned
addresses that are never read."""
import ctypes
import re

import pytest
import torch

from paper_2607_21224_amd import cpdp, q8
from paper_2607_21224_amd.build import ROOT

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                reason="fake device addresses: CPU-only module")

OK, INVALID, NULL, MISALIGNED, OVERLAP, DTYPE, TOO_LARGE = (
    cpdp.CPDP_OK, cpdp.CPDP_ERR_INVALID_ARG, cpdp.CPDP_ERR_NULL, cpdp.CPDP_ERR_MISALIGNED,
    cpdp.CPDP_ERR_OVERLAP, cpdp.CPDP_ERR_DTYPE, cpdp.CPDP_ERR_TOO_LARGE)
F32, BF16 = cpdp.CPDP_F32, cpdp.CPDP_BF16


def at(k):
    return (1 << 40) + (k << 36)


def test_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(f"{ROOT}/include/cpdp_q8.h").read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(cpdp_q8_\w+)\s*\(", text)))
    assert names == sorted(q8.EXPORTS)
    lib = ctypes.CDLL(q8.LIB_PATH)
    for n in names:
        assert hasattr(lib, n), n


# Every call with arguments that would be accepted; T (M) is the only thing a
# test of refusals leaves in place.
CALLS = {
    "cpdp_q8_rows": dict(x=at(0), ldx=64, x_dt=BF16, T=8, D=64, q=at(1), ldq=64, scale=at(2),
                         y=at(3), ldy=64, y_dt=BF16, stream=None),
    "cpdp_q8_values": dict(q=at(1), ldq=64, scale=at(2), T=8, D=64, y=at(3), ldy=64, y_dt=F32,
                           stream=None),
    "cpdp_q8_norm": dict(x=at(0), ldx=64, residual=at(1), ldr=64, act_dt=BF16, w=at(2), w_dt=F32,
                         eps=1e-6, T=8, D=64, h=at(3), ldh=64, q=at(4), ldq=64, scale=at(5),
                         rstd=at(6), y=at(7), ldy=64, y_dt=BF16, stream=None),
    "cpdp_q8_norm_bwd": dict(dy=at(0), lddy=64, h=at(1), ldh=64, dres=at(2), lddres=64,
                             act_dt=BF16, w=at(3), w_dt=F32, rstd=at(4), T=8, D=64, dx=at(5),
                             lddx=64, dw=at(6), dw_dt=F32, workspace=at(7),
                             workspace_bytes=1 << 20, stream=None),
    "cpdp_q8_matmul": dict(a=at(0), lda=64, a_scale=at(1), b=at(2), ldb=64, b_scale=at(3), M=8,
                           N=32, K=64, y=at(4), ldy=32, y_dt=BF16, workspace=at(5),
                           workspace_bytes=1 << 30, stream=None),
    "cpdp_q8_act": dict(kind=1, g=at(0), u=at(1), ldg=64, act_dt=BF16, T=8, F=64, q=at(2), ldq=64,
                        scale=at(3), y=at(4), ldy=64, y_dt=BF16, cg=at(5), cg_scale=at(6),
                        cu=at(7), cu_scale=at(8), ldc=64, stream=None),
    "cpdp_q8_act_bwd": dict(kind=1, da=at(0), ldda=64, act_dt=BF16, cg=at(1), cg_scale=at(2),
                            cu=at(3), cu_scale=at(4), ldc=64, T=8, F=64, dg=at(5), du=at(6),
                            lddg=64, stream=None),
    "cpdp_q8_grad_input": dict(dy=at(0), lddy=32, dy_dt=BF16, b=at(1), ldb=64, b_scale=at(2), T=80,
                               N=32, K=64, dx=at(3), lddx=64, out_dt=F32, workspace=at(4),
                               workspace_bytes=1 << 30, stream=None),
    "cpdp_q8_grad_weight": dict(dy=at(0), lddy=32, dy_dt=BF16, a=at(1), lda=64, a_scale=at(2),
                                T=80, N=32, K=64, dw=at(3), lddw=64, out_dt=F32, workspace=at(4),
                                workspace_bytes=1 << 30, stream=None),
}
ROWS = {n: "M" if n == "cpdp_q8_matmul" else "T" for n in CALLS}
OPTIONAL = {"y", "rstd", "dres"}
POINTERS = {n: [k for k, v in a.items() if isinstance(v, int) and v >= 1 << 40]
            for n, a in CALLS.items()}
STRIDES = {n: [k for k in a if k.startswith("ld")] for n, a in CALLS.items()}
TYPES = {n: [k for k in a if k.endswith("_dt")] for n, a in CALLS.items()}


def call(name, **change):
    args = dict(CALLS[name])
    assert set(change) <= set(args)
    args.update(change)
    return getattr(q8.lib, name)(*args.values())


@pytest.mark.parametrize("name", CALLS)
def test_counts(name):
    assert call(name, **{ROWS[name]: -1}) == INVALID
    assert call(name, **{ROWS[name]: 1 << 31}) == INVALID
    inner = "D" if "D" in CALLS[name] else "F" if "F" in CALLS[name] else "K"
    assert call(name, **{inner: 0}) == INVALID
    assert call(name, **{inner: -4}) == INVALID
    assert call(name, **{inner: 65}) == INVALID  # past the row stride


@pytest.mark.parametrize("name,which", [
    (n, k) for n in CALLS for k in POINTERS[n] if (n, k) != ("cpdp_q8_matmul", "workspace")])
def test_pointers(name, which):
    if which not in OPTIONAL:
        assert call(name, **{which: None}) == NULL
    step = 2 if "scale" in which or which == "rstd" else 8
    assert call(name, **{which: CALLS[name][which] + step}) == MISALIGNED
    assert call(name, **{which: (1 << 64) - 16}) == INVALID  # runs past the address space


@pytest.mark.parametrize("name,which", [(n, k) for n in CALLS for k in STRIDES[n]])
def test_strides(name, which):
    assert call(name, **{which: 16}) == INVALID
    assert call(name, **{which: 68 + 1}) == MISALIGNED
    assert call(name, **{which: -64}) == INVALID
    assert call(name, **{which: 1 << 29}) == INVALID


@pytest.mark.parametrize("name,which", [(n, k) for n in CALLS for k in TYPES[n]])
def test_storage_types(name, which):
    assert call(name, **{which: 2}) == DTYPE
    assert call(name, **{which: -1}) == DTYPE


WRITTEN = {"cpdp_q8_rows": "q scale y", "cpdp_q8_values": "y", "cpdp_q8_norm": "h q scale rstd y",
           "cpdp_q8_norm_bwd": "dx dw workspace", "cpdp_q8_matmul": "y workspace",
           "cpdp_q8_act": "q scale y cg cg_scale cu cu_scale", "cpdp_q8_act_bwd": "dg du",
           "cpdp_q8_grad_input": "dx workspace", "cpdp_q8_grad_weight": "dw workspace"}


@pytest.mark.parametrize("name,out,other", [
    (n, o, k) for n in CALLS for o in WRITTEN[n].split() for k in POINTERS[n]
    if o != k and (n, o, k) not in {("cpdp_q8_norm", "h", "x"), ("cpdp_q8_norm", "h", "residual")}
    and "workspace" not in (o, k)])
def test_overlaps(name, out, other):
    """An output on the last bytes of another buffer."""
    args = CALLS[name]
    # 8 rows of at least 32 bytes lie between the first byte and this one
    assert call(name, **{out: args[other] + 16}) == OVERLAP


def test_norm_in_place_means_the_very_same_rows():
    n = "cpdp_q8_norm"
    x = CALLS[n]["x"]
    assert call(n, h=x + 16) == OVERLAP
    assert call(n, h=x, ldh=128) == OVERLAP
    assert call(n, h=None) == NULL and call(n, residual=None) == NULL
    for eps in (-1.0, float("nan"), float("inf")):
        assert call(n, eps=eps) == INVALID


@pytest.mark.parametrize("name", [n for n in CALLS if "workspace" in CALLS[n]])
def test_workspaces(name):
    a = CALLS[name]
    sizes = {"cpdp_q8_norm_bwd": ("T", "D"), "cpdp_q8_matmul": ("M", "N", "K")}.get(
        name, ("T", "N", "K", "dy_dt", "out_dt"))
    # a product whose sum is cut into slices has a workspace too
    big = dict(K=4096, lda=4096, ldb=4096) if name == "cpdp_q8_matmul" else {}
    need = getattr(q8.lib, name + "_workspace")(*[{**a, **big}[k] for k in sizes])
    if need > 0:
        assert call(name, **big, workspace_bytes=need - 1) == INVALID
        assert call(name, **big, workspace=None) == NULL
        out = WRITTEN[name].split()[0]
        assert call(name, **big, workspace=a[out]) == OVERLAP


def test_rows_that_a_tile_cannot_address():
    assert call("cpdp_q8_matmul", lda=1 << 23) == TOO_LARGE
    assert call("cpdp_q8_matmul", K=131072, lda=131072, ldb=131072) == INVALID
    assert call("cpdp_q8_grad_input", N=1 << 22, lddy=1 << 22, T=1) == TOO_LARGE
    assert call("cpdp_q8_grad_weight", T=1 << 22) == TOO_LARGE


@pytest.mark.parametrize("kind", [-1, 2])
def test_unknown_activation(kind):
    assert call("cpdp_q8_act", kind=kind) == INVALID
    assert call("cpdp_q8_act_bwd", kind=kind) == INVALID


@pytest.mark.parametrize("name", [n for n in CALLS
                                  if n not in ("cpdp_q8_norm_bwd", "cpdp_q8_grad_weight")])
def test_no_rows(name):
    """Nothing to do: OK without a launch, pointers of empty matrices included."""
    rows = {"x", "residual", "h", "q", "scale", "rstd", "a", "a_scale", "g", "u", "cg", "cg_scale",
            "cu", "cu_scale", "da", "dg", "du", "dy", "dx", "y"}
    gone = {k: None for k in POINTERS[name] if k in rows}
    if name == "cpdp_q8_norm":
        gone = {k: v for k, v in gone.items() if k not in ("residual", "h")}
    assert call(name, **{ROWS[name]: 0}) == OK
    if name != "cpdp_q8_act":
        assert call(name, **{ROWS[name]: 0}, **gone) == OK


def test_python_checks_come_first():
    x = torch.zeros(4, 32)
    q, s = torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4)
    with pytest.raises(ValueError, match="current GPU"):
        q8.cpdp_q8_rows(x, q, s)
    with pytest.raises(ValueError, match="float32 or torch.bfloat16"):
        q8.cpdp_q8_rows(x.half(), q, s)


@pytest.mark.parametrize("kind", [1 << 32, -(1 << 40) + 1, 1 << 80])
def test_python_refuses_numbers_no_activation_has(kind):
    x = torch.zeros(4, 32)
    q, s = torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4)
    with pytest.raises(ValueError, match="kind"):
        q8.cpdp_q8_act(kind, x, q=q, scale=s)
    with pytest.raises(ValueError, match="kind"):
        q8.cpdp_q8_act_bwd(kind, x, q, s, x)
