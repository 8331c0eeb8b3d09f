"""Python binding of the 8-bit activation path's C ABI (include/cpdp_q8.h).

Argument marshalling only: the operators run in the gfx950 kernels of
``libcpdp_q8.so``, and importing this module without it raises ImportError.  The
functions carry the C names.  They take torch tensors and read sizes, row
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

from .cpdp import CPDP_BF16, CPDP_F32, CPDP_OK, CpdpError
from .state import _on, round_up

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libcpdp_q8.so")

CPDP_Q8_MAX_K = 131071
CPDP_ACT_GELU = 0
CPDP_ACT_SWIGLU = 1
ACTIVATIONS = {"gelu": CPDP_ACT_GELU, "swiglu": CPDP_ACT_SWIGLU}

# every symbol declared in include/cpdp_q8.h
EXPORTS = ("cpdp_q8_rows", "cpdp_q8_values", "cpdp_q8_norm", "cpdp_q8_norm_bwd_workspace",
           "cpdp_q8_norm_bwd", "cpdp_q8_matmul_workspace", "cpdp_q8_matmul", "cpdp_q8_act",
           "cpdp_q8_act_bwd", "cpdp_q8_grad_input_workspace", "cpdp_q8_grad_input",
           "cpdp_q8_grad_weight_workspace", "cpdp_q8_grad_weight")


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load a build of the library and declare its signatures (torch is
    imported first, so that its HIP runtime is the one that is used)."""
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
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = n if name.endswith("_workspace") else i
    return lib


lib = load_library()

_CODE = {torch.float32: CPDP_F32, torch.bfloat16: CPDP_BF16}


def empty_rows(T: int, D: int, dtype, device="cuda") -> torch.Tensor:
    """An uninitialised (T, D) matrix whose rows start on 16-byte boundaries."""
    step = 16 // torch.empty((), dtype=dtype).element_size()
    return torch.empty((T, round_up(max(D, 1), step)), dtype=dtype, device=device)[:, :D]


def _fail(name, what):
    raise ValueError(f"{name}: {what}")


def _place(x, name):
    """A tensor's address; it has to be on the current GPU."""
    if not x.is_cuda or x.get_device() != torch.cuda.current_device():
        _fail(name, f"a tensor on the current GPU expected, this one is on {x.device}")
    return x.data_ptr()


def _mat(x, name, shape=None, dtype=None):
    """(address, row stride) of a matrix argument."""
    if x.dim() != 2 or (shape is not None and x.shape != shape):
        want = "a matrix" if shape is None else f"shape {tuple(shape)}"
        _fail(name, f"{want} expected, the tensor is {tuple(x.shape)}")
    if dtype is not None and x.dtype is not dtype:
        _fail(name, f"{dtype} expected, the tensor is {x.dtype}")
    rows, cols = x.shape
    ld, step = x.stride()
    if step != 1 and cols > 1:
        _fail(name, f"rows have to be dense, their elements are {step} apart")
    if rows <= 1:  # no second row: any aligned stride does
        ld = round_up(max(cols, 1), 16)
    return _place(x, name), ld


def _float_mat(x, name, shape=None):
    """(address, row stride, storage code) of an fp32 or bf16 matrix."""
    dt = _CODE.get(x.dtype)
    if dt is None:
        _fail(name, f"torch.float32 or torch.bfloat16 expected, the tensor is {x.dtype}")
    p, ld = _mat(x, name, shape)
    return p, ld, dt


def _vec(x, name, n, dtype=torch.float32):
    if x.dim() != 1 or x.shape[0] != n or (n > 1 and x.stride(0) != 1):
        _fail(name, f"a dense vector of {n} expected, the tensor is {tuple(x.shape)}")
    if dtype is not None and x.dtype is not dtype:
        _fail(name, f"{dtype} expected, the tensor is {x.dtype}")
    return _place(x, name)


def _float_vec(x, name, n):
    dt = _CODE.get(x.dtype)
    if dt is None:
        _fail(name, f"torch.float32 or torch.bfloat16 expected, the tensor is {x.dtype}")
    return _vec(x, name, n, None), dt


def _scratch(workspace, need, stream, device):
    """(address, bytes, tensor to keep) of a call's workspace."""
    if workspace is None:
        if need == 0:
            return None, 0, None
        if stream is not None:
            _fail("workspace", "needed where a stream is given")
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    elif not workspace.is_contiguous():
        _fail("workspace", "a contiguous tensor expected")
    return _place(workspace, "workspace"), workspace.nbytes, workspace


def _done(status, where, check):
    if check and status != CPDP_OK:
        raise CpdpError(status, where)
    return status


def _kind(kind):
    if isinstance(kind, str):
        if kind not in ACTIVATIONS:
            _fail("kind", f"one of {sorted(ACTIVATIONS)} expected, got {kind!r}")
        return ACTIVATIONS[kind]
    return int(kind)


def cpdp_q8_rows(x, q, scale, y=None, stream=None, check=True):
    """Hold the rows of x in 8 bits (and write their values to y)."""
    xp, ldx, dt = _float_mat(x, "x")
    T, D = x.shape
    qp, ldq = _mat(q, "q", x.shape, torch.int8)
    yp, ldy, ydt = (None, 0, CPDP_F32) if y is None else _float_mat(y, "y", x.shape)
    s = lib.cpdp_q8_rows(xp, ldx, dt, T, D, qp, ldq, _vec(scale, "scale", T), yp, ldy, ydt,
                         _stream(stream))
    return _done(s, "cpdp_q8_rows", check)


def cpdp_q8_values(q, scale, y, stream=None, check=True):
    """Read 8-bit rows back into y."""
    qp, ldq = _mat(q, "q", None, torch.int8)
    T, D = q.shape
    yp, ldy, dt = _float_mat(y, "y", q.shape)
    s = lib.cpdp_q8_values(qp, ldq, _vec(scale, "scale", T), T, D, yp, ldy, dt, _stream(stream))
    return _done(s, "cpdp_q8_values", check)


def cpdp_q8_norm(x, w, eps, q, scale, residual=None, h=None, rstd=None, y=None, stream=None,
                 check=True):
    """h <- x + residual; q, scale <- its root-mean-square norm, times w, in 8
    bits; rstd for the backward pass and the values y where they are given."""
    xp, ldx, dt = _float_mat(x, "x")
    shape = x.shape
    T, D = shape
    wp, wdt = _float_vec(w, "w", D)
    qp, ldq = _mat(q, "q", shape, torch.int8)
    rp = hp = None
    ldr = ldh = 0
    if residual is not None:
        rp, ldr = _mat(residual, "residual", shape, x.dtype)
    if h is not None:
        hp, ldh = _mat(h, "h", shape, x.dtype)
    yp, ldy, ydt = (None, 0, CPDP_F32) if y is None else _float_mat(y, "y", shape)
    s = lib.cpdp_q8_norm(xp, ldx, rp, ldr, dt, wp, wdt, eps, T, D, hp, ldh, qp, ldq,
                         _vec(scale, "scale", T), None if rstd is None else _vec(rstd, "rstd", T),
                         yp, ldy, ydt, _stream(stream))
    return _done(s, "cpdp_q8_norm", check)


def cpdp_q8_norm_bwd_workspace(T, D) -> int:
    return lib.cpdp_q8_norm_bwd_workspace(T, D)


def cpdp_q8_norm_bwd(dy, h, w, rstd, dx, dw, dres=None, workspace=None, stream=None, check=True):
    """dx and dw from dy (and the gradient dres that reaches h beside it)."""
    dyp, lddy, dt = _float_mat(dy, "dy")
    shape = dy.shape
    T, D = shape
    hp, ldh = _mat(h, "h", shape, dy.dtype)
    rp, ldr = (None, 0) if dres is None else _mat(dres, "dres", shape, dy.dtype)
    wp, wdt = _float_vec(w, "w", D)
    dxp, lddx = _mat(dx, "dx", shape, dy.dtype)
    dwp, dwdt = _float_vec(dw, "dw", D)
    wsp, n, keep = _scratch(workspace, lib.cpdp_q8_norm_bwd_workspace(T, D), stream, dy.device)
    s = lib.cpdp_q8_norm_bwd(dyp, lddy, hp, ldh, rp, ldr, dt, wp, wdt, _vec(rstd, "rstd", T), T, D,
                             dxp, lddx, dwp, dwdt, wsp, n, _stream(stream))
    return _done(s, "cpdp_q8_norm_bwd", check)


def cpdp_q8_matmul_workspace(M, N, K) -> int:
    return lib.cpdp_q8_matmul_workspace(M, N, K)


def cpdp_q8_matmul(a, a_scale, b, b_scale, y, workspace=None, stream=None, check=True):
    """y <- a b^T, scaled by a's and b's rows."""
    ap, lda = _mat(a, "a", None, torch.int8)
    M, K = a.shape
    bp, ldb = _mat(b, "b", None, torch.int8)
    N = b.shape[0]
    if b.shape[1] != K:
        _fail("b", f"{K} columns expected, the tensor is {tuple(b.shape)}")
    yp, ldy, dt = _float_mat(y, "y", (M, N))
    wsp, n, keep = _scratch(workspace, lib.cpdp_q8_matmul_workspace(M, N, K), stream, a.device)
    s = lib.cpdp_q8_matmul(ap, lda, _vec(a_scale, "a_scale", M), bp, ldb,
                           _vec(b_scale, "b_scale", N), M, N, K, yp, ldy, dt, wsp, n,
                           _stream(stream))
    return _done(s, "cpdp_q8_matmul", check)


def cpdp_q8_act(kind, g, u=None, *, q, scale, y=None, cg=None, sg=None, cu=None, su=None,
                stream=None, check=True):
    """q, scale <- the activation of g (and u) in 8 bits, y its values; cg, sg
    and cu, su <- g and u in 8 bits, the checkpoint."""
    k = _kind(kind)
    gp, ldg, dt = _float_mat(g, "g")
    shape = g.shape
    T, F = shape
    up = None
    if k == CPDP_ACT_SWIGLU:
        if u is None:
            _fail("u", "swiglu takes two inputs")
        up, ldu = _mat(u, "u", shape, g.dtype)
        if ldu != ldg:
            _fail("u", f"the row stride of g, {ldg}, expected; it is {ldu}")
    elif u is not None or cu is not None or su is not None:
        _fail("u", "gelu takes one input")
    qp, ldq = _mat(q, "q", shape, torch.int8)
    yp, ldy, ydt = (None, 0, CPDP_F32) if y is None else _float_mat(y, "y", shape)
    cgp = cup = None
    ldc = 0
    if cg is not None:
        cgp, ldc = _mat(cg, "cg", shape, torch.int8)
    if cu is not None:
        cup, ldcu = _mat(cu, "cu", shape, torch.int8)
        if cg is None or ldcu != ldc:
            _fail("cu", "the row stride of cg expected")
    s = lib.cpdp_q8_act(k, gp, up, ldg, dt, T, F, qp, ldq, _vec(scale, "scale", T), yp, ldy, ydt,
                        cgp, None if sg is None else _vec(sg, "sg", T), cup,
                        None if su is None else _vec(su, "su", T), ldc, _stream(stream))
    return _done(s, "cpdp_q8_act", check)


def cpdp_q8_act_bwd(kind, da, cg, sg, dg, cu=None, su=None, du=None, stream=None, check=True):
    """dg (and du) from da and the checkpoint."""
    k = _kind(kind)
    dap, ldda, dt = _float_mat(da, "da")
    shape = da.shape
    T, F = shape
    cgp, ldc = _mat(cg, "cg", shape, torch.int8)
    dgp, lddg = _mat(dg, "dg", shape, da.dtype)
    cup = sup = dup = None
    if k == CPDP_ACT_SWIGLU:
        if cu is None or su is None or du is None:
            _fail("cu", "swiglu takes cu, su and du")
        cup, ldcu = _mat(cu, "cu", shape, torch.int8)
        dup, lddu = _mat(du, "du", shape, da.dtype)
        if ldcu != ldc or lddu != lddg:
            _fail("du", "the row strides of cg and dg expected for cu and du")
        sup = _vec(su, "su", T)
    elif cu is not None or su is not None or du is not None:
        _fail("cu", "gelu takes one input")
    s = lib.cpdp_q8_act_bwd(k, dap, ldda, dt, cgp, _vec(sg, "sg", T), cup, sup, ldc, T, F, dgp, dup,
                            lddg, _stream(stream))
    return _done(s, "cpdp_q8_act_bwd", check)


def cpdp_q8_grad_input_workspace(T, N, K, dy_dtype, out_dtype) -> int:
    return lib.cpdp_q8_grad_input_workspace(T, N, K, _CODE[dy_dtype], _CODE[out_dtype])


def cpdp_q8_grad_weight_workspace(T, N, K, dy_dtype, out_dtype) -> int:
    return lib.cpdp_q8_grad_weight_workspace(T, N, K, _CODE[dy_dtype], _CODE[out_dtype])


def cpdp_q8_grad_input(dy, b, b_scale, dx, workspace=None, stream=None, check=True):
    """dx <- dy b, with b's rows scaled."""
    dyp, lddy, dt = _float_mat(dy, "dy")
    T, N = dy.shape
    bp, ldb = _mat(b, "b", None, torch.int8)
    K = b.shape[1]
    if b.shape[0] != N:
        _fail("b", f"{N} rows expected, the tensor is {tuple(b.shape)}")
    dxp, lddx, odt = _float_mat(dx, "dx", (T, K))
    wsp, n, keep = _scratch(workspace, lib.cpdp_q8_grad_input_workspace(T, N, K, dt, odt), stream,
                            dy.device)
    s = lib.cpdp_q8_grad_input(dyp, lddy, dt, bp, ldb, _vec(b_scale, "b_scale", N), T, N, K, dxp,
                               lddx, odt, wsp, n, _stream(stream))
    return _done(s, "cpdp_q8_grad_input", check)


def cpdp_q8_grad_weight(dy, a, a_scale, dw, workspace=None, stream=None, check=True):
    """dw <- dy^T a, with a's rows scaled."""
    dyp, lddy, dt = _float_mat(dy, "dy")
    T, N = dy.shape
    ap, lda = _mat(a, "a", None, torch.int8)
    K = a.shape[1]
    if a.shape[0] != T:
        _fail("a", f"{T} rows expected, the tensor is {tuple(a.shape)}")
    dwp, lddw, odt = _float_mat(dw, "dw", (N, K))
    wsp, n, keep = _scratch(workspace, lib.cpdp_q8_grad_weight_workspace(T, N, K, dt, odt), stream,
                            dy.device)
    s = lib.cpdp_q8_grad_weight(dyp, lddy, dt, ap, lda, _vec(a_scale, "a_scale", T), T, N, K, dwp,
                                lddw, odt, wsp, n, _stream(stream))
    return _done(s, "cpdp_q8_grad_weight", check)


def _stream(stream):
    s = _on(stream)
    return s if s is None or isinstance(s, int) else s.cuda_stream
