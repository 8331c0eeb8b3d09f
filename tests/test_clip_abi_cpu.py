"""What gradient norms and clipping refuse, on the host before any GPU work.  Fake aligned
addresses that are never read; only calls that fail validation are made."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from paper_2607_21224_amd import build, cpdp

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                reason="fake device addresses: CPU-only module")

G, N, WS = 1 << 40, 2 << 40, 3 << 40
GOOD = dict(grads=G, W=4, P=1000, ld=1024, grad_dt=0, flags=0, norm=N, ws=WS, nbytes=1 << 20,
            max_norm=1.0)
INF, NAN = float("inf"), float("nan")


def norm(**kw):
    a = {**GOOD, **kw}
    return cpdp.lib.cpdp_grad_norm(a["grads"], a["W"], a["P"], a["ld"], a["grad_dt"], a["flags"],
                                   a["norm"], a["ws"], a["nbytes"], None)


def clip(**kw):
    a = {**GOOD, **kw}
    return cpdp.lib.cpdp_clip_grads(a["grads"], a["W"], a["P"], a["ld"], a["grad_dt"],
                                    a["max_norm"], a["flags"], a["norm"], a["ws"], a["nbytes"],
                                    None)


@pytest.mark.parametrize("fn", [norm, clip])
@pytest.mark.parametrize("kw,status", [
    (dict(W=0), cpdp.CPDP_ERR_INVALID_ARG), (dict(W=-1), cpdp.CPDP_ERR_INVALID_ARG),
    (dict(W=(1 << 23) + 1, P=1, ld=4, nbytes=1 << 40), cpdp.CPDP_ERR_INVALID_ARG),
    (dict(P=-1), cpdp.CPDP_ERR_INVALID_ARG), (dict(ld=999), cpdp.CPDP_ERR_INVALID_ARG),
    (dict(P=1 << 58, ld=1 << 58), cpdp.CPDP_ERR_INVALID_ARG),
    (dict(flags=2), cpdp.CPDP_ERR_INVALID_ARG), (dict(flags=3), cpdp.CPDP_ERR_INVALID_ARG),
    (dict(grad_dt=2), cpdp.CPDP_ERR_DTYPE), (dict(grad_dt=-1), cpdp.CPDP_ERR_DTYPE),
    (dict(grads=None), cpdp.CPDP_ERR_NULL), (dict(norm=None), cpdp.CPDP_ERR_NULL),
    (dict(ws=None), cpdp.CPDP_ERR_NULL), (dict(nbytes=0), cpdp.CPDP_ERR_INVALID_ARG),
    (dict(grads=G + 4), cpdp.CPDP_ERR_MISALIGNED), (dict(ld=1001), cpdp.CPDP_ERR_MISALIGNED),
    (dict(ld=1004, grad_dt=1), cpdp.CPDP_ERR_MISALIGNED),
    (dict(norm=N + 2), cpdp.CPDP_ERR_MISALIGNED), (dict(ws=WS + 8), cpdp.CPDP_ERR_MISALIGNED),
    (dict(norm=G + 4 * 1023), cpdp.CPDP_ERR_OVERLAP), (dict(norm=G - 12), cpdp.CPDP_ERR_OVERLAP),
    (dict(ws=G + 16), cpdp.CPDP_ERR_OVERLAP), (dict(ws=N), cpdp.CPDP_ERR_OVERLAP),
    (dict(grads=2 ** 64 - 4096), cpdp.CPDP_ERR_INVALID_ARG)])
def test_refusals(fn, kw, status):
    assert fn(**kw) == status


@pytest.mark.parametrize("x", [0.0, -1.0, INF, -INF, NAN])
def test_bad_max_norm(x):
    assert clip(max_norm=x) == cpdp.CPDP_ERR_INVALID_ARG
    assert cpdp.lib.cpdp_clip_grads_plan(None, x, 0, N, WS, 1 << 20, None) != cpdp.CPDP_OK


def test_a_short_workspace():
    for W, P in ((1, 1), (4, 1000), (8, 23712932), (3000, 5), (1, 0)):
        need = cpdp.cpdp_grad_norm_workspace(W, P)
        assert need >= 8 * W
        kw = dict(W=W, P=P, ld=(P + 7) // 8 * 8, nbytes=need - 1)
        assert norm(**kw) == clip(**kw) == cpdp.CPDP_ERR_INVALID_ARG


def test_workspace_of_what_is_refused():
    for W, P in ((0, 5), (-1, 5), (4, -1), ((1 << 23) + 1, 5), (1, 1 << 58)):
        assert cpdp.cpdp_grad_norm_workspace(W, P) == 0
    assert cpdp.lib.cpdp_grad_norm_plan_workspace(None) == 0


def test_plans():
    """Only a handle that a build filled is taken."""
    lib = cpdp.lib
    call = lambda p: (lib.cpdp_grad_norm_plan(p, 0, N, WS, 1 << 20, None),  # noqa: E731
                      lib.cpdp_clip_grads_plan(p, 1.0, 0, N, WS, 1 << 20, None))
    assert call(None) == (cpdp.CPDP_ERR_NULL,) * 2
    p = cpdp.cpdp_plan()
    assert call(ctypes.byref(p)) == (cpdp.CPDP_ERR_NULL,) * 2
    p.table, p.W, p.n_tensors, p.total_chunks, p.total_numel, p.seal = G, 4, 3, 10, 999, 12345
    assert call(ctypes.byref(p)) == (cpdp.CPDP_ERR_INVALID_ARG,) * 2
    assert lib.cpdp_grad_norm_plan_workspace(ctypes.byref(p)) == 0


def test_the_binding_checks_tensors():
    g, n, ws = torch.zeros(4, 1024), torch.zeros(4), torch.zeros(1 << 20, dtype=torch.uint8)
    with pytest.raises(ValueError, match="device tensors"):
        cpdp.cpdp_grad_norm(g, 4, 1000, 1024, N, WS)
    with pytest.raises(ValueError, match="grads"):
        cpdp.cpdp_clip_grads(g[:3], 4, 1000, 1024, 1.0, N, WS)
    with pytest.raises(ValueError, match="grads"):
        cpdp.cpdp_grad_norm(g, 4, 1000, 1024, N, WS, "bf16")
    with pytest.raises(ValueError, match="norm"):
        cpdp.cpdp_grad_norm(G, 4, 1000, 1024, n[:3], WS)
    with pytest.raises(ValueError, match="device tensors"):
        cpdp.cpdp_grad_norm(G, 4, 1000, 1024, N, ws)
    with pytest.raises(cpdp.CpdpError):  # an address without its size
        cpdp.cpdp_grad_norm(G, 4, 1000, 1024, N, None)


ROOT = build.ROOT


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_validation_under_sanitizers(tmp_path):
    """The validation layer for the host, with calls that pass and calls that do not."""
    exe = str(tmp_path / "clip_driver")
    native, csrc = os.path.join(ROOT, "tests", "native"), os.path.join(build.PKG, "csrc")
    r = subprocess.run(["g++", "-std=c++17", "-Wall", "-fsanitize=address,undefined",
                        "-fno-sanitize-recover=all", "-g", "-I", os.path.join(ROOT, "include"),
                        "-I", csrc, os.path.join(csrc, "clip_api.cpp"),
                        os.path.join(csrc, "cpdp_api.cpp"), os.path.join(native, "stub_launch.cpp"),
                        os.path.join(native, "clip_driver.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "OK", r.stdout + r.stderr
