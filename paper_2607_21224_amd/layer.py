"""The MLP half of a transformer block on the 8-bit activation path, trained by the
CPDP steps.

``Q8Mlp`` holds no weights: they are slices of a replica's row of
``CpdpState.params``, and its gradients go into the same slices of a row of
gradients, so one model of any number of such layers is one row.  What a layer's
forward pass keeps for its backward pass (``Saved``) is one byte an activation, a
quarter of fp32 and half of bf16, but for the sum that the norm is taken of; what
passes need for a while (``Scratch``), layers whose passes run one after the
other share::

    mlp = Q8Mlp(dim=384, hidden=1536)
    st = CpdpState(W=8, P=mlp.numel, K=4)
    st.init(theta0)                            # (P,) fp32: mlp.init(generator)
    grads = torch.zeros((8, st.ld), device="cuda")
    saved = mlp.saved(tokens)
    for t in range(1, T + 1):
        for i in range(8):
            mlp.forward(st.params[i], x[i], saved)     # saved.y
            dy = ...                                   # the loss' gradient of saved.y
            mlp.backward(st.params[i], dy, saved, grads[i])
        st.step(t, grads, hyper, T)

For dim 384, hidden 1536, GELU and bf16, bytes a token: n, z and a in 8 bits 3456, their
scales and rstd 16, h 768, and the results y and dx 768 each, once a layer; z, da and dn
6912, once for all that share them.  (h, n, z and a in bf16 are 7680.)  Replicas that run
one after the other, as here, need one ``Saved`` a layer, not one each.

Forward, with `8(.)` for rounding to 8-bit rows (cpdp_q8.h):
    h = x + residual;  n = 8(norm(h) * w);  z = n 8(W1)^T;  a = 8(act(z))
    y = a 8(W2)^T
The gated kind's two inner products are one, of twice the channels: their weights follow
each other in a row, and g and u are the halves of z.
Backward passes gradients through the roundings unchanged, and uses the rounded
operands.
"""
from __future__ import annotations

import torch

from . import q8
from .state import round_up

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}


class Scratch:
    """What passes over `T` tokens need for a while: the inner product's result and its
    gradient (z), the gradients of the activation (da) and of the norm (dn), and the
    operators' workspace.  Nothing of it outlives a pass, so layers of one shape may share
    one where no two of their passes run at the same time (one stream)."""

    def __init__(self, mlp: "Q8Mlp", T: int, device="cuda"):
        self.T, self.shape = T, mlp.shape
        self.z_all = q8.empty_rows(T, mlp.inner, mlp.act_dtype, device)
        self.da = q8.empty_rows(T, mlp.hidden, mlp.act_dtype, device)
        self.dn = q8.empty_rows(T, mlp.dim, mlp.act_dtype, device)
        self.workspace = torch.empty(mlp.workspace_bytes(T), dtype=torch.uint8, device=device)


class Saved:
    """What a forward pass over `T` tokens leaves for its backward pass, and the results of
    both; it serves one replica after another.  `scratch`: a Scratch to share."""

    def __init__(self, mlp: "Q8Mlp", T: int, device="cuda", scratch: Scratch | None = None):
        def rows(r, c, dt=mlp.act_dtype):
            return q8.empty_rows(r, c, dt, device)

        def vec(n):
            return torch.empty(n, device=device)

        if scratch is None:
            scratch = Scratch(mlp, T, device)
        elif (scratch.T, scratch.shape) != (T, mlp.shape):
            raise ValueError(f"scratch: made for {scratch.T} tokens of a layer {scratch.shape}, "
                             f"this one is for {T} of {mlp.shape}")
        D, F, i8 = mlp.dim, mlp.hidden, torch.int8
        halves = range(0, mlp.inner, F)
        self.T = T
        # one byte an activation: the norm's output, the activation's inputs and
        # output, and the weights as they were used
        self.n, self.n_scale, self.rstd = rows(T, D, i8), vec(T), vec(T)
        self.cg, self.g_scale = rows(T, F, i8), vec(T)
        self.cu, self.u_scale = (rows(T, F, i8), vec(T)) if mlp.gated else (None, None)
        self.a, self.a_scale = rows(T, F, i8), vec(T)
        q, scale = self.w_in = rows(mlp.inner, D, i8), vec(mlp.inner)
        self.w1 = [(q[i:i + F], scale[i:i + F]) for i in halves]
        self.w2 = rows(D, F, i8), vec(D)
        # the sum that the norm is taken of, and the results
        self.h, self.y, self.dx = rows(T, D), rows(T, D), rows(T, D)
        self.z_all, self.da, self.dn = scratch.z_all, scratch.da, scratch.dn
        self.z = [self.z_all[:, i:i + F] for i in halves]
        self.workspace = scratch.workspace


class Q8Mlp:
    """dim -> hidden -> dim with a root-mean-square norm before it; kind "gelu", or
    "swiglu" with two inner products."""

    def __init__(self, dim: int, hidden: int, kind: str = "gelu", eps: float = 1e-6,
                 act_dt: str = "bf16"):
        if kind not in q8.ACTIVATIONS:
            raise ValueError(f"kind must be one of {sorted(q8.ACTIVATIONS)}, got {kind!r}")
        if act_dt not in _DT:
            raise ValueError(f"act_dt must be 'f32' or 'bf16', got {act_dt!r}")
        if dim % 8 or hidden % 8:
            raise ValueError("dim and hidden must be multiples of 8: the weights' rows lie one "
                             "after the other in a replica's row, each on a 16-byte boundary")
        self.dim, self.hidden, self.kind, self.eps = int(dim), int(hidden), kind, float(eps)
        self.gated = kind == "swiglu"
        self.inner = self.hidden * (2 if self.gated else 1)  # channels of z
        self.shape = (self.dim, self.hidden, kind, act_dt)
        self.act_dtype = _DT[act_dt]
        shapes = [("norm", (dim,)), ("w1", (hidden, dim))]
        if self.gated:
            shapes.append(("w1u", (hidden, dim)))
        shapes.append(("w2", (dim, hidden)))
        self.tensors, at = {}, 0
        for name, shape in shapes:
            n = shape[0] * (shape[1] if len(shape) == 2 else 1)
            self.tensors[name] = (at, shape)
            at = round_up(at + n, 8)
        self.numel = at

    def view(self, row: torch.Tensor, name: str) -> torch.Tensor:
        """A tensor of the layer in a replica's row of parameters or gradients."""
        at, shape = self.tensors[name]
        n = shape[0] * (shape[1] if len(shape) == 2 else 1)
        return row[at:at + n].view(shape)

    def _w_in(self, row: torch.Tensor) -> torch.Tensor:
        """The inner product's weights, (inner, dim): w1, and w1u after it."""
        at, _ = self.tensors["w1"]
        return row[at:at + self.inner * self.dim].view(self.inner, self.dim)

    def init(self, generator: torch.Generator | None = None, device="cuda") -> torch.Tensor:
        """Initial parameters, (numel,) fp32: the norm's weight 1, the others normal
        with the variance 1 / inputs."""
        row = torch.zeros(self.numel, device=device)
        self.view(row, "norm").fill_(1.0)
        for name, (_, shape) in self.tensors.items():
            if len(shape) == 2:
                self.view(row, name).normal_(0.0, shape[1] ** -0.5, generator=generator)
        return row

    def saved(self, T: int, device="cuda", scratch: Scratch | None = None) -> Saved:
        return Saved(self, int(T), device, scratch)

    def scratch(self, T: int, device="cuda") -> Scratch:
        return Scratch(self, int(T), device)

    def workspace_bytes(self, T: int) -> int:
        """The largest workspace of the layer's calls over T tokens."""
        D, F, I, dt = self.dim, self.hidden, self.inner, self.act_dtype
        need = [q8.cpdp_q8_matmul_workspace(T, I, D), q8.cpdp_q8_matmul_workspace(T, D, F),
                q8.cpdp_q8_norm_bwd_workspace(T, D)]
        for N, K in ((I, D), (D, F)):
            need.append(q8.cpdp_q8_grad_input_workspace(T, N, K, dt, dt))
            need += [q8.cpdp_q8_grad_weight_workspace(T, N, K, dt, g) for g in _DT.values()]
        return max(need + [16])

    def forward(self, params, x, saved: Saved, residual=None, stream=None) -> torch.Tensor:
        """saved.y <- the layer's output for x (T, dim); params is a replica's row.
        With a residual saved.h is x + residual, the residual of what follows; without one
        the backward pass reads x again, which has to stay as it is until then."""
        s = saved
        if residual is None:
            q8.cpdp_q8_norm(x, self.view(params, "norm"), self.eps, q=s.n, scale=s.n_scale,
                            rstd=s.rstd, stream=stream)
            s.norm_of = x
        else:
            q8.cpdp_q8_norm(x, self.view(params, "norm"), self.eps, q=s.n, scale=s.n_scale,
                            rstd=s.rstd, residual=residual, h=s.h, stream=stream)
            s.norm_of = s.h
        q8.cpdp_q8_rows(self._w_in(params), *s.w_in, stream=stream)
        q8.cpdp_q8_matmul(s.n, s.n_scale, *s.w_in, s.z_all, workspace=s.workspace, stream=stream)
        q8.cpdp_q8_act(self.kind, *s.z, q=s.a, scale=s.a_scale, cg=s.cg, sg=s.g_scale, cu=s.cu,
                       su=s.u_scale, stream=stream)
        q8.cpdp_q8_rows(self.view(params, "w2"), *s.w2, stream=stream)
        q8.cpdp_q8_matmul(s.a, s.a_scale, *s.w2, s.y, workspace=s.workspace, stream=stream)
        return s.y

    def backward(self, params, dy, saved: Saved, grads, dres=None, stream=None) -> torch.Tensor:
        """The gradients of the last forward pass over `saved`, of the parameters
        into `grads` (a replica's row) and of the input, returned; dres is what
        reaches x + residual past the layer."""
        s = saved
        kw = {"workspace": s.workspace, "stream": stream}
        q8.cpdp_q8_grad_weight(dy, s.a, s.a_scale, self.view(grads, "w2"), **kw)
        q8.cpdp_q8_grad_input(dy, *s.w2, s.da, **kw)
        # z is done with: its gradient takes its place
        q8.cpdp_q8_act_bwd(self.kind, s.da, s.cg, s.g_scale, s.z[0], cu=s.cu, su=s.u_scale,
                           du=s.z[1] if self.gated else None, stream=stream)
        q8.cpdp_q8_grad_weight(s.z_all, s.n, s.n_scale, self._w_in(grads), **kw)
        q8.cpdp_q8_grad_input(s.z_all, *s.w_in, s.dn, **kw)
        q8.cpdp_q8_norm_bwd(s.dn, s.norm_of, self.view(params, "norm"), s.rstd, s.dx,
                            self.view(grads, "norm"), dres=dres, **kw)
        return s.dx
