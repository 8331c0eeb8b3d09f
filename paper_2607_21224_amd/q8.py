"""Python binding of the 8-bit activation path's C ABI (include/cpdp_q8.h).

Argument marshalling only: the operators run in the gfx950 kernels of
``libcpdp_q8.so``, which the extension module ``_q8`` calls; importing this module
without them raises ImportError.  The functions carry the C names.  They take torch tensors and read sizes, row
strides and storage types off them:

* a matrix argument is a 2-D tensor whose rows are dense (``stride(1) == 1``);
  rows start on 16-byte boundaries (``empty_rows`` allocates such a tensor for
  any number of columns, and a slice of its columns or rows is one too);
* 8-bit rows are an int8 matrix and an fp32 vector of scales;
* results are written into tensors that the caller passes.

``stream`` is a ``torch.cuda.Stream``, a raw ``hipStream_t`` integer, or None for
torch's current stream.  ``workspace`` is a contiguous tensor of at least the
bytes that the matching ``*_workspace`` function returns; None takes one from
torch's allocator for the call, which is possible on the current stream only.
A wrong shape, type or device raises ValueError before the library is called; a
non-zero status of the library raises ``cpdp.CpdpError`` (``check=False`` returns
it instead).
"""
from __future__ import annotations

import ctypes
import os

import torch

from .cpdp import CPDP_BF16, CPDP_F32, CpdpError
from .state import round_up

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libcpdp_q8.so")

CPDP_Q8_MAX_K = 131071
CPDP_Q8_MAX_T = 2097088
CPDP_ACT_GELU = 0
CPDP_ACT_SWIGLU = 1
ACTIVATIONS = {"gelu": CPDP_ACT_GELU, "swiglu": CPDP_ACT_SWIGLU}

# every symbol declared in include/cpdp_q8.h
EXPORTS = ("cpdp_q8_rows", "cpdp_q8_values", "cpdp_q8_norm", "cpdp_q8_norm_bwd_workspace",
           "cpdp_q8_norm_bwd", "cpdp_q8_matmul_workspace", "cpdp_q8_matmul", "cpdp_q8_act",
           "cpdp_q8_act_bwd", "cpdp_q8_grad_input_workspace", "cpdp_q8_grad_input",
           "cpdp_q8_grad_weight_workspace", "cpdp_q8_grad_weight", "cpdp_q8_xent_workspace",
           "cpdp_q8_xent", "cpdp_q8_xent_bwd_workspace", "cpdp_q8_xent_bwd",
           "cpdp_q8_xent_miss", "cpdp_q8_xent_miss_bwd")


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load a build of the library and declare its signatures, for callers with
    raw addresses (torch is imported first, so that its HIP runtime is the one
    that is used)."""
    if not os.path.exists(path):
        raise ImportError(f"{path} is not built; run `python -m paper_2607_21224_amd.build` "
                          "(the 8-bit path has no CPU fallback)")
    lib = ctypes.CDLL(path)
    p, i, n, f = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float
    sig = {
        "cpdp_q8_rows": [p, n, i, n, n, p, n, p, p, n, i, p],
        "cpdp_q8_values": [p, n, p, n, n, p, n, i, p],
        "cpdp_q8_norm": [p, n, p, n, i, p, i, f, n, n, p, n, p, n, p, p, p, n, i, p],
        "cpdp_q8_norm_bwd_workspace": [n, n],
        "cpdp_q8_norm_bwd": [p, n, p, n, p, n, i, p, i, p, n, n, p, n, p, i, p, n, p],
        "cpdp_q8_matmul_workspace": [n, n, n],
        "cpdp_q8_matmul": [p, n, p, p, n, p, n, n, n, p, n, i, p, n, p],
        "cpdp_q8_act": [i, p, p, n, i, n, n, p, n, p, p, n, i, p, p, p, p, n, p],
        "cpdp_q8_act_bwd": [i, p, n, i, p, p, p, p, n, n, n, p, p, n, p],
        "cpdp_q8_grad_input_workspace": [n, n, n, i, i],
        "cpdp_q8_grad_input": [p, n, i, p, n, p, n, n, n, p, n, i, p, n, p],
        "cpdp_q8_grad_weight_workspace": [n, n, n, i, i],
        "cpdp_q8_grad_weight": [p, n, i, p, n, p, n, n, n, p, n, i, p, n, p],
        "cpdp_q8_xent_workspace": [n, n, n],
        "cpdp_q8_xent": [p, n, p, p, n, p, p, n, n, n, p, p, p, n, p],
        "cpdp_q8_xent_bwd_workspace": [n, n, n, i, i],
        "cpdp_q8_xent_bwd": [p, n, p, p, n, p, p, p, p, n, n, n, p, n, i, p, n, i, p, n, p],
        "cpdp_q8_xent_miss": [p, n, p, p, n, p, p, n, n, n, p, p, p, p, n, p],
        "cpdp_q8_xent_miss_bwd": [p, n, p, p, n, p, p, p, p, p, n, n, n, p, n, i, p, n, i, p, n, p],
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = n if name.endswith("_workspace") else i
    return lib


lib = load_library()

from . import _q8  # noqa: E402  (after torch, whose libraries it uses)

_CODE = {torch.float32: CPDP_F32, torch.bfloat16: CPDP_BF16}


def empty_rows(T: int, D: int, dtype, device="cuda") -> torch.Tensor:
    """An uninitialised (T, D) matrix whose rows start on 16-byte boundaries."""
    step = 16 // torch.empty((), dtype=dtype).element_size()
    return torch.empty((T, round_up(max(D, 1), step)), dtype=dtype, device=device)[:, :D]


def _stream(stream):
    return stream if stream is None or isinstance(stream, int) else stream.cuda_stream


def _done(status, where, check):
    if check and status:
        raise CpdpError(status, where)
    return status


def _kind(kind):
    if isinstance(kind, str):
        if kind not in ACTIVATIONS:
            raise ValueError(f"kind: one of {sorted(ACTIVATIONS)} expected, got {kind!r}")
        return ACTIVATIONS[kind]
    return int(kind)


def cpdp_q8_rows(x, q, scale, y=None, stream=None, check=True):
    """Hold the rows of x in 8 bits (and write their values to y)."""
    return _done(_q8.rows(x, q, scale, y, _stream(stream)), "cpdp_q8_rows", check)


def cpdp_q8_values(q, scale, y, stream=None, check=True):
    """Read 8-bit rows back into y."""
    return _done(_q8.values(q, scale, y, _stream(stream)), "cpdp_q8_values", check)


def cpdp_q8_norm(x, w, eps, q, scale, residual=None, h=None, rstd=None, y=None, stream=None,
                 check=True):
    """h <- x + residual; q, scale <- its root-mean-square norm, times w, in 8
    bits; rstd for the backward pass and the values y where they are given."""
    s = _q8.norm(x, w, eps, q, scale, residual, h, rstd, y, _stream(stream))
    return _done(s, "cpdp_q8_norm", check)


def cpdp_q8_norm_bwd_workspace(T, D) -> int:
    return lib.cpdp_q8_norm_bwd_workspace(T, D)


def cpdp_q8_norm_bwd(dy, h, w, rstd, dx, dw, dres=None, workspace=None, stream=None, check=True):
    """dx and dw from dy (and the gradient dres that reaches h beside it)."""
    s = _q8.norm_bwd(dy, h, w, rstd, dx, dw, dres, workspace, _stream(stream))
    return _done(s, "cpdp_q8_norm_bwd", check)


def cpdp_q8_matmul_workspace(M, N, K) -> int:
    return lib.cpdp_q8_matmul_workspace(M, N, K)


def cpdp_q8_matmul(a, a_scale, b, b_scale, y, workspace=None, stream=None, check=True):
    """y <- a b^T, scaled by a's and b's rows."""
    s = _q8.matmul(a, a_scale, b, b_scale, y, workspace, _stream(stream))
    return _done(s, "cpdp_q8_matmul", check)


def cpdp_q8_act(kind, g, u=None, *, q, scale, y=None, cg=None, sg=None, cu=None, su=None,
                stream=None, check=True):
    """q, scale <- the activation of g (and u) in 8 bits, y its values; cg, sg
    and cu, su <- g and u in 8 bits, the checkpoint.  kind: "gelu" or "swiglu"."""
    s = _q8.act(_kind(kind), g, u, q, scale, y, cg, sg, cu, su, _stream(stream))
    return _done(s, "cpdp_q8_act", check)


def cpdp_q8_act_bwd(kind, da, cg, sg, dg, cu=None, su=None, du=None, stream=None, check=True):
    """dg (and du) from da and the checkpoint."""
    s = _q8.act_bwd(_kind(kind), da, cg, sg, dg, cu, su, du, _stream(stream))
    return _done(s, "cpdp_q8_act_bwd", check)


def cpdp_q8_grad_input_workspace(T, N, K, dy_dtype, out_dtype) -> int:
    return lib.cpdp_q8_grad_input_workspace(T, N, K, _CODE[dy_dtype], _CODE[out_dtype])


def cpdp_q8_grad_weight_workspace(T, N, K, dy_dtype, out_dtype) -> int:
    return lib.cpdp_q8_grad_weight_workspace(T, N, K, _CODE[dy_dtype], _CODE[out_dtype])


def cpdp_q8_grad_input(dy, b, b_scale, dx, workspace=None, stream=None, check=True):
    """dx <- dy b, with b's rows scaled."""
    s = _q8.grad_input(dy, b, b_scale, dx, workspace, _stream(stream))
    return _done(s, "cpdp_q8_grad_input", check)


def cpdp_q8_grad_weight(dy, a, a_scale, dw, workspace=None, stream=None, check=True):
    """dw <- dy^T a, with a's rows scaled."""
    s = _q8.grad_weight(dy, a, a_scale, dw, workspace, _stream(stream))
    return _done(s, "cpdp_q8_grad_weight", check)


def cpdp_q8_xent_workspace(T, V, K) -> int:
    return lib.cpdp_q8_xent_workspace(T, V, K)


def cpdp_q8_xent(x, x_scale, w, w_scale, target, loss, lse, workspace=None, stream=None,
                 check=True, miss=None):
    """lse, loss <- the softmax cross entropy of the logits x w^T (rows of both scaled) and
    target, (T,) int64; tokens whose target is negative do not count.  miss, (T,), if given:
    1 - exp(-loss), for the gradients (cpdp_q8_xent_miss)."""
    s = _q8.xent(x, x_scale, w, w_scale, target, loss, lse, miss, workspace, _stream(stream))
    return _done(s, "cpdp_q8_xent", check)


def cpdp_q8_xent_bwd_workspace(T, V, K, dx_dtype, dw_dtype) -> int:
    """(the type of a gradient that is left out does not matter: that of the other)"""
    return lib.cpdp_q8_xent_bwd_workspace(T, V, K, _CODE[dx_dtype], _CODE[dw_dtype])


def cpdp_q8_xent_bwd(x, x_scale, w, w_scale, target, lse, g, dx=None, dw=None, workspace=None,
                     stream=None, check=True, miss=None):
    """dx, dw (the ones that are given) <- the gradients of x's and w's values, where g (T,)
    is the gradient of the loss and lse is cpdp_q8_xent's; with its miss, those of tokens of
    small loss are as exact as the loss (cpdp_q8_xent_miss_bwd)."""
    s = _q8.xent_bwd(x, x_scale, w, w_scale, target, lse, miss, g, dx, dw, workspace,
                     _stream(stream))
    return _done(s, "cpdp_q8_xent_bwd", check)
