"""The 8-bit activation path of a transformer layer, as measurable cases.

W replicas of a model on one GPU keep W sets of activations there, so what a
layer keeps between its forward and its backward pass is held in 8 bits: rows
of int8 with one scale each.  A row is written as

    s = the smallest bfloat16 number >= 2^-126 with 127 s >= max |x|
    q = x / s, rounded to the nearest whole number, ties to even

and stands for s q.  A pass is one operator on such rows.

Fields of a case
  op   norm      residual's addition, root-mean-square norm, 8-bit rows
       norm_bwd  its backward pass: the input's and the weight's gradient
       product   product of 8-bit rows with 8-bit weights
       act       activation of a layer's inner product: forward pass with 8-bit
                 output and 8-bit checkpoint, then the backward pass from it
       grads     the product's backward pass from its 8-bit operands: gradients
                 of the input and of the weights
  T    rows (tokens)
  N    product, grads: output channels;   K    input channels
  D    norm: channels;   F    act: channels of the activation's output
  kind act: gelu, or swiglu (silu of one input times the other)
  res  norm, norm_bwd: with a residual (its gradient)
  dt   type of the activations and gradients: f32 or bf16
"""
from __future__ import annotations

import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}
_EPS = 1e-6
_SMALLEST = 2.0 ** -126  # scale of a row of zeros


def listed():
    return [
        # one token of a serving loop: the call itself is what it costs
        {"name": "norm_one_token", "op": "norm", "T": 1, "D": 4096, "res": True, "dt": "bf16"},
        # 8 images of 197 tokens through a ViT-S block (dim 384), fp32 as its
        # replicas are trained
        {"name": "norm_vit", "op": "norm", "T": 1576, "D": 384, "res": True, "dt": "f32"},
        # a batch of long sequences on a wide layer
        {"name": "norm_long", "op": "norm", "T": 16384, "D": 8192, "res": True, "dt": "bf16"},
        {"name": "norm_bwd_vit", "op": "norm_bwd", "T": 1576, "D": 384, "res": True, "dt": "f32"},
        {"name": "norm_bwd_long", "op": "norm_bwd", "T": 8192, "D": 4096, "res": True,
         "dt": "bf16"},
        # one token through a square layer: the weights are read once
        {"name": "product_one_token", "op": "product", "T": 1, "N": 4096, "K": 4096,
         "dt": "bf16"},
        # no dimension a multiple of a tile: a ViT-S block's inputs with a
        # class token's channels appended
        {"name": "product_ragged", "op": "product", "T": 1576, "N": 1153, "K": 385, "dt": "f32"},
        # a batch of long sequences through a wide layer
        {"name": "product_large", "op": "product", "T": 8192, "N": 8192, "K": 8192, "dt": "bf16"},
        # a ViT-S block's MLP (384 x 4 channels)
        {"name": "act_vit", "op": "act", "kind": "gelu", "T": 1576, "F": 1536, "dt": "f32"},
        # a wide gated layer
        {"name": "act_gated_large", "op": "act", "kind": "swiglu", "T": 8192, "F": 8192,
         "dt": "bf16"},
        # a ViT-S block's first MLP product
        {"name": "grads_vit", "op": "grads", "T": 1576, "N": 1536, "K": 384, "dt": "f32"},
        # a wide layer's second product
        {"name": "grads_large", "op": "grads", "T": 8192, "N": 8192, "K": 4096, "dt": "bf16"},
    ]


def draw(rng):
    """Sizes spread over their logarithm, half of them odd ones; a fifth of the
    cases are a few tokens."""
    def size(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        if rng.random() < 0.5:
            n = (n + 15) // 16 * 16
        return max(lo, min(hi, n))

    op = rng.choice(["norm", "norm_bwd", "product", "act", "grads"])
    most = 16384 if op in ("norm", "norm_bwd") else 8192
    T = rng.randint(1, 64) if rng.random() < 0.2 else size(1, most)
    c = {"op": op, "T": T}
    if op in ("norm", "norm_bwd"):
        c.update(D=size(32, 8192), res=rng.random() < 0.7)
    elif op == "act":
        c.update(F=size(32, 8192), kind=rng.choice(["gelu", "swiglu"]))
    else:
        c.update(N=size(32, 8192), K=size(32, 8192 if op == "product" else 4096))
    c["dt"] = rng.choice(["f32", "bf16"])
    return c


def work(case):
    e, T, op = _BYTES[case["dt"]], case["T"], case["op"]
    if op == "norm":
        D = case["D"]
        # input, 8-bit rows, their values in bf16, and with a residual that and the sum
        n = T * D * (e + 1 + 2 + (2 * e if case["res"] else 0))
        return {"bytes": n + 8 * T + 4 * D, "flops": 8 * T * D}
    if op == "norm_bwd":
        D = case["D"]
        return {"bytes": T * D * e * (4 if case["res"] else 3) + 4 * T + 8 * D,
                "flops": 9 * T * D}
    if op == "act":
        nz = 2 if case["kind"] == "swiglu" else 1
        F = case["F"]
        fwd = T * F * (e * nz + nz + 1 + 2) + 4 * T * (nz + 1)
        bwd = T * F * (e + nz + e * nz) + 4 * T * nz
        return {"bytes": fwd + bwd, "flops": 40 * T * F}
    N, K = case["N"], case["K"]
    if op == "product":
        return {"bytes": T * K + N * K + 4 * (T + N) + T * N * e, "flops": 2 * T * N * K}
    return {"bytes": T * N * e + (T + N) * K * (1 + e) + 4 * (T + N), "flops": 4 * T * N * K}


def _up16(n):
    return (n + 15) // 16 * 16


def _rows(gen, T, D, dt, scale=None):
    """(T, D) values ~ N(0, 1) times scale[D], in rows padded to 16 elements."""
    x = torch.randn((T, _up16(D)), generator=gen, device="cuda")[:, :D]
    if scale is not None:
        x = x * scale
    full = torch.empty((T, _up16(D)), dtype=_DT[dt], device="cuda")
    full[:, :D] = x
    return full[:, :D]


def _blank(T, D, dtype):
    return torch.empty((T, _up16(D)), dtype=dtype, device="cuda")[:, :D]


def _channels(gen, D):
    """Sizes of the channels of an activation: mostly alike, one in 64 some ten
    times as large."""
    c = torch.exp(0.3 * torch.randn(D, generator=gen, device="cuda"))
    return torch.where(torch.rand(D, generator=gen, device="cuda") < 1 / 64, 10 * c, c)


def _row_scale(amax):
    """The smallest bfloat16 number s >= 2^-126 with 127 s >= amax (fp32)."""
    low = (amax / 127).contiguous().view(torch.int32) & -65536
    s = low.view(torch.float32)
    up = (low + 65536).view(torch.float32)
    return torch.where(s * 127 < amax, up, s).clamp_min(_SMALLEST)


def _quantised(x):
    """8-bit rows of x (fp32), as whole numbers in fp32, and their scales."""
    s = _row_scale(x.abs().amax(-1))
    return torch.round(x / s[:, None]), s


def _held(gen, T, D, scale=None):
    """Rows that an earlier operator left in 8 bits."""
    q, s = _quantised(_rows(gen, T, D, "f32", scale))
    full = torch.zeros((T, _up16(D)), dtype=torch.int8, device="cuda")
    full[:, :D] = q.to(torch.int8)
    return full[:, :D], s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    c, T, dt = dict(case), case["T"], case["dt"]
    st = {"case": c}
    if c["op"] in ("norm", "norm_bwd"):
        D = c["D"]
        ch = _channels(gen, D)
        st["w"] = 1 + 0.1 * torch.randn(D, generator=gen, device="cuda")
        if c["op"] == "norm":
            st["x"] = _rows(gen, T, D, dt, ch)
            st["res"] = _rows(gen, T, D, dt, ch) if c["res"] else None
            st["out"] = {"h": _blank(T, D, _DT[dt]) if c["res"] else None,
                         "q": _blank(T, D, torch.int8), "scale": torch.empty(T, device="cuda"),
                         "rstd": torch.empty(T, device="cuda"),
                         "y": _blank(T, D, torch.bfloat16)}
        else:
            st["h"] = _rows(gen, T, D, dt, ch)
            st["rstd"] = torch.rsqrt(st["h"].float().square().mean(-1) + _EPS)
            st["dy"] = _rows(gen, T, D, dt)
            st["dres"] = _rows(gen, T, D, dt) if c["res"] else None
            st["out"] = {"dx": _blank(T, D, _DT[dt]), "dw": torch.empty(D, device="cuda")}
    elif c["op"] == "act":
        F = c["F"]
        gated = c["kind"] == "swiglu"
        ch = _channels(gen, F)
        st["g"] = _rows(gen, T, F, dt, ch)
        st["u"] = _rows(gen, T, F, dt) if gated else None
        st["da"] = _rows(gen, T, F, dt)
        empty = lambda: torch.empty(T, device="cuda")  # noqa: E731
        st["out"] = {"q": _blank(T, F, torch.int8), "scale": empty(),
                     "y": _blank(T, F, torch.bfloat16),
                     "cg": _blank(T, F, torch.int8), "sg": empty(),
                     "cu": _blank(T, F, torch.int8) if gated else None,
                     "su": empty() if gated else None,
                     "dg": _blank(T, F, _DT[dt]),
                     "du": _blank(T, F, _DT[dt]) if gated else None}
    else:
        N, K = c["N"], c["K"]
        st["a"], st["sa"] = _held(gen, T, K, _channels(gen, K))
        st["b"], st["sb"] = _held(gen, N, K, torch.full((K,), K ** -0.5, device="cuda"))
        if c["op"] == "product":
            st["out"] = {"y": _blank(T, N, _DT[dt])}
        else:
            st["dy"] = _rows(gen, T, N, dt)
            st["out"] = {"dx": _blank(T, K, _DT[dt]), "dw": _blank(N, K, _DT[dt])}
    return st


def run(state):
    return (_own if own else _plain)(state)


def _own(st):
    """The calls of the framework's operators."""
    from paper_2607_21224_amd import q8
    c, o = st["case"], st["out"]
    if c["op"] == "norm":
        q8.cpdp_q8_norm(st["x"], st["w"], _EPS, q=o["q"], scale=o["scale"], residual=st["res"],
                        h=o["h"], rstd=o["rstd"], y=o["y"])
        return {"h": o["h"], "y": o["y"], "rstd": o["rstd"]}
    if c["op"] == "norm_bwd":
        q8.cpdp_q8_norm_bwd(st["dy"], st["h"], st["w"], st["rstd"], o["dx"], o["dw"],
                            dres=st["dres"])
        return o
    if c["op"] == "product":
        q8.cpdp_q8_matmul(st["a"], st["sa"], st["b"], st["sb"], o["y"])
        return o
    if c["op"] == "act":
        q8.cpdp_q8_act(c["kind"], st["g"], st["u"], q=o["q"], scale=o["scale"], y=o["y"],
                       cg=o["cg"], sg=o["sg"], cu=o["cu"], su=o["su"])
        q8.cpdp_q8_act_bwd(c["kind"], st["da"], o["cg"], o["sg"], o["dg"], cu=o["cu"],
                           su=o["su"], du=o["du"])
        return {"y": o["y"], "dg": o["dg"], "du": o["du"]}
    q8.cpdp_q8_grad_input(st["dy"], st["b"], st["sb"], o["dx"])
    q8.cpdp_q8_grad_weight(st["dy"], st["a"], st["sa"], o["dw"])
    return o


def _plain(st):
    c = st["case"]
    dt = _DT[c["dt"]]
    if c["op"] == "norm":
        x, w = st["x"], st["w"]
        h = (x.float() + st["res"].float()).to(dt) if c["res"] else x
        hf = h.float()
        rstd = torch.rsqrt((hf * hf).mean(-1) + _EPS)
        q, s = _quantised(hf * rstd[:, None] * w)
        return {"h": h if c["res"] else None, "y": (q * s[:, None]).to(torch.bfloat16),
                "rstd": rstd}
    if c["op"] == "norm_bwd":
        n = st["h"].float() * st["rstd"][:, None]
        dy = st["dy"].float()
        dn = dy * st["w"]
        dx = (dn - n * (dn * n).mean(-1, keepdim=True)) * st["rstd"][:, None]
        if c["res"]:
            dx = dx + st["dres"].float()
        return {"dx": dx.to(dt), "dw": (dy * n).sum(0)}
    if c["op"] == "act":
        g, da = st["g"].float(), st["da"].float()
        gated = c["kind"] == "swiglu"
        if gated:
            a = g * torch.sigmoid(g) * st["u"].float()
        else:
            a = 0.5 * g * (1 + torch.erf(g * math.sqrt(0.5)))
        q, s = _quantised(a)
        y = (q * s[:, None]).to(torch.bfloat16)
        cg, sg = _quantised(g)
        G = cg * sg[:, None]
        if gated:
            cu, su = _quantised(st["u"].float())
            sig = torch.sigmoid(G)
            dg = da * (cu * su[:, None]) * sig * (1 + G * (1 - sig))
            return {"y": y, "dg": dg.to(dt), "du": (da * G * sig).to(dt)}
        cdf = 0.5 * (1 + torch.erf(G * math.sqrt(0.5)))
        pdf = torch.exp(-0.5 * G * G) * (1 / math.sqrt(2 * math.pi))
        return {"y": y, "dg": (da * (cdf + G * pdf)).to(dt), "du": None}
    a = st["a"].float() * st["sa"][:, None]
    b = st["b"].float() * st["sb"][:, None]
    if c["op"] == "product":
        return {"y": (a @ b.t()).to(dt)}
    dy = st["dy"].float()
    return {"dx": (dy @ b).to(dt), "dw": (dy.t() @ a).to(dt)}


def exact(case, seed):
    """The definitions in 64 bits: sums as products with vectors, the scale by
    its bits."""
    st = prepare(case, seed)
    up = lambda t: t.to(torch.float64)  # noqa: E731
    c = st["case"]

    def held(v):
        top = v.abs().max(dim=1).values
        # the quotient by a tensor is correctly rounded, then up to 8 significant
        # bits: the last 45 of the double's 52 are cleared
        bits = (top / torch.full_like(top, 127.0)).view(torch.int64)
        s = (((bits + (1 << 45) - 1) >> 45) << 45).view(torch.float64)
        s = torch.maximum(s, torch.full_like(s, _SMALLEST)).unsqueeze(1)
        return torch.round(v / s) * s

    if c["op"] == "norm":
        h = up(st["x"])
        if c["res"]:
            h = up((h + up(st["res"])).to(_DT[c["dt"]]))
        r = 1.0 / torch.sqrt(torch.linalg.vector_norm(h, dim=1) ** 2 / c["D"] + _EPS)
        return {"h": h if c["res"] else None, "y": held(h * torch.outer(r, up(st["w"]))),
                "rstd": r}
    if c["op"] == "norm_bwd":
        r, w, dy = up(st["rstd"]).unsqueeze(1), up(st["w"]), up(st["dy"])
        n = up(st["h"]) * r
        t = (dy * n) @ w / c["D"]
        dx = r * (dy * w - n * t.unsqueeze(1))
        return {"dx": dx + up(st["dres"]) if c["res"] else dx,
                "dw": torch.ones(c["T"], dtype=torch.float64, device="cuda") @ (dy * n)}
    if c["op"] == "act":
        g, da = up(st["g"]), up(st["da"])
        G = held(g)
        if c["kind"] == "swiglu":
            u = up(st["u"])
            e = torch.exp(-G)
            dsilu = (1 + e + G * e) / (1 + e) ** 2
            # exp(-G) past the largest double: the derivative there is 0
            dsilu = torch.where(torch.isfinite(dsilu), dsilu, torch.zeros_like(dsilu))
            return {"y": held(u * g / (1 + torch.exp(-g))), "dg": da * held(u) * dsilu,
                    "du": da * G / (1 + e)}
        phi = lambda t: 0.5 * torch.erfc(-t / math.sqrt(2.0))  # noqa: E731
        return {"y": held(g * phi(g)), "du": None,
                "dg": da * (phi(G) + G * torch.exp(-(G ** 2) / 2) / math.sqrt(2 * math.pi))}
    a, b = up(st["a"]), up(st["b"])
    sa, sb = up(st["sa"]), up(st["sb"])
    if c["op"] == "product":
        return {"y": torch.outer(sa, sb) * torch.mm(a, b.t().contiguous())}
    dy = up(st["dy"])
    return {"dx": torch.mm(dy * sb, b), "dw": torch.mm((dy * sa.unsqueeze(1)).t(), a)}
