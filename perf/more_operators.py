"""What stands between a layer's output and a replica's step, as measurable cases: the
loss with its gradient, and the gradient's norm with clipping.

The loss is the softmax cross entropy of T rows over V classes, both held in 8 bits (rows of
int8 with a scale each, as the 8-bit activation path leaves them), without the T x V logits
being kept.  With z[t, v] = xs[t] ws[v] sum_k x[t, k] w[v, k]:

    lse[t]   = log sum_v exp z[t, v]
    loss[t]  = lse[t] - z[t, target[t]],  0 where target[t] < 0 (padding)
    d[t, v]  = g[t] (exp(z[t, v] - lse[t]) - [v = target[t]]),  0 where target[t] < 0
    dx[t, k] = sum_v d[t, v] ws[v] w[v, k]
    dw[v, k] = sum_t d[t, v] xs[t] x[t, k]

Clipping takes the norm over all coordinates of a replica's gradient (or of the mean of the
W replicas' gradients) and scales what is longer than max_norm:

    c = min(1, max_norm / (norm + 1e-6)),  grad <- c grad

Fields of a case
  op    score  lse and loss (evaluation, scoring of tokens)
        train  lse and loss, then dx and dw
        norm   norms of the gradients
        clip   norms, and the gradients scaled in place
  T     score, train: rows (tokens, images);  V  classes;  K  channels
  dx    train: type of dx, f32 or bf16;  dw  of dw
  W     norm, clip: replicas;  P  coordinates of each
  n     tensors that a replica's gradient is held as (0: one flat row)
  dt    type of the gradients
  mean  norm of the replicas' mean gradient, not of each replica's
  long  clip: every gradient is longer than max_norm, not about half of them
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}
_MAX_NORM = 1.0
_IGNORED = -100


def listed():
    return [
        # one token scored against a vocabulary: the weights are read once
        {"name": "score_one_token", "op": "score", "T": 1, "V": 32768, "K": 4096},
        # an evaluation batch, no dimension a multiple of a tile
        {"name": "score_ragged", "op": "score", "T": 1003, "V": 50001, "K": 1025},
        # evaluation of long sequences over a large vocabulary
        {"name": "score_large", "op": "score", "T": 8192, "V": 131072, "K": 2048},
        # a batch of 128 images through a ViT-S head (384 channels, 100 classes), fp32 as
        # its replicas are trained
        {"name": "train_classes", "op": "train", "T": 128, "V": 100, "K": 384, "dx": "f32",
         "dw": "f32"},
        # a small model's vocabulary, odd sizes, fp32
        {"name": "train_ragged", "op": "train", "T": 997, "V": 12345, "K": 385, "dx": "f32",
         "dw": "f32"},
        # bf16 activations and fp32 gradient rows, a middling model with a large vocabulary
        {"name": "train_mixed", "op": "train", "T": 4096, "V": 65536, "K": 1024, "dx": "bf16",
         "dw": "f32"},
        # a wide model, all bf16
        {"name": "train_large", "op": "train", "T": 8192, "V": 32768, "K": 4096, "dx": "bf16",
         "dw": "bf16"},
        # the tiny workload's rows: a launch or two is what it costs
        {"name": "norm_tiny", "op": "norm", "W": 4, "P": 262144, "n": 0, "dt": "f32",
         "mean": False},
        # what a synchronised step of ResNet-50-sized replicas clips by, bf16 rows
        {"name": "norm_mean", "op": "norm", "W": 16, "P": 23917832, "n": 0, "dt": "bf16",
         "mean": True},
        # two replicas of a small model
        {"name": "clip_small", "op": "clip", "W": 2, "P": 10007, "n": 0, "dt": "f32",
         "mean": False, "long": True},
        # ViT-S-sized replicas, each by its own norm
        {"name": "clip_rows", "op": "clip", "W": 8, "P": 21332068, "n": 0, "dt": "f32",
         "mean": False, "long": True},
        # ResNet-50-sized replicas held as 161 tensors each
        {"name": "clip_tensors", "op": "clip", "W": 8, "P": 23712932, "n": 161, "dt": "f32",
         "mean": False, "long": True},
    ]


def draw(rng):
    """Sizes spread over their logarithm, half of them odd ones; some losses are of a few
    tokens, or of a few classes."""
    def size(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        if rng.random() < 0.5:
            n = (n + 15) // 16 * 16
        return max(lo, min(hi, n))

    op = rng.choice(["score", "train", "train", "norm", "clip", "clip"])
    if op in ("score", "train"):
        T = rng.randint(1, 64) if rng.random() < 0.25 else size(1, 8192)
        V = rng.randint(2, 200) if rng.random() < 0.2 else size(2, 131072)
        K = size(8, min(4096, 8192 * 131072 * 1024 // (T * V)))
        c = {"op": op, "T": T, "V": V, "K": K}
        if op == "train":
            c.update(dx=rng.choice(["f32", "bf16"]), dw=rng.choice(["f32", "bf16"]))
        return c
    W = rng.choice([1, 2, 3, 4, 5, 8, 12, 16, 32])
    n = rng.choice([0, 0, rng.randint(1, 300)])
    P = size(max(1, n), 8 * 23712932 // W)
    c = {"op": op, "W": W, "P": P, "n": n, "dt": "f32" if n else rng.choice(["f32", "bf16"]),
         "mean": rng.random() < 0.4}
    if op == "clip":
        c["long"] = rng.random() < 0.5
    return c


def work(case):
    if case["op"] in ("score", "train"):
        T, V, K = case["T"], case["V"], case["K"]
        n = (T + V) * (K + 4) + 8 * T + 8 * T
        if case["op"] == "score":
            return {"bytes": n, "flops": 2 * T * V * K}
        n += 4 * T + K * (T * _BYTES[case["dx"]] + V * _BYTES[case["dw"]])
        return {"bytes": n, "flops": 6 * T * V * K}
    n = case["W"] * case["P"] * _BYTES[case["dt"]]
    if case["op"] == "clip" and case["long"]:
        n *= 2
    elif case["op"] == "clip":
        n = n * 3 // 2
    return {"bytes": n, "flops": 2 * case["W"] * case["P"]}


def _up(n, m):
    return (n + m - 1) // m * m


# ---- inputs -----------------------------------------------------------------------

def _held(x):
    """Rows of x (fp32) in 8 bits: the smallest bfloat16 scale s >= 2^-126 with
    127 s >= max |x|, and x / s rounded to whole numbers."""
    amax = x.abs().amax(-1)
    low = (amax / 127).contiguous().view(torch.int32) & -65536
    s = low.view(torch.float32)
    s = torch.where(s * 127 < amax, (low + 65536).view(torch.float32), s).clamp_min(2.0 ** -126)
    full = torch.zeros((x.shape[0], _up(x.shape[1], 16)), dtype=torch.int8, device="cuda")
    full[:, :x.shape[1]] = torch.round(x / s[:, None]).to(torch.int8)
    return full[:, :x.shape[1]], s


def _blank(R, C, dtype):
    return torch.empty((R, _up(C, 16)), dtype=dtype, device="cuda")[:, :C]


def _loss_inputs(case, gen):
    """Weights of logits of a few units; targets by a steep distribution, some rows padding;
    rows that lean towards their target's weights, from not at all to where the target has
    nearly all of the probability."""
    T, V, K = case["T"], case["V"], case["K"]
    rand = lambda *s: torch.rand(s, generator=gen, device="cuda")  # noqa: E731
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    w = randn(V, K) * K ** -0.5
    target = (V * rand(T) ** 3).long().clamp_max(V - 1)
    x = randn(T, K) * torch.exp(0.3 * randn(K))
    x = x + 12 * rand(T, 1) * w[target]
    target[rand(T) < 0.06] = _IGNORED
    st = {}
    st["x"], st["xs"] = _held(x)
    st["w"], st["ws"] = _held(w)
    st["target"] = target
    st["loss"], st["lse"] = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    if case["op"] == "train":
        # the gradient of the mean over the tokens that count
        st["g"] = (1.0 / (target >= 0).sum().clamp_min(1).float()).expand(T).contiguous()
        st["dx"] = _blank(T, K, _DT[case["dx"]])
        st["dw"] = _blank(V, K, _DT[case["dw"]])
    return st


def _r50(classes):
    """Elements of the 161 tensors of ResNet-50 (7 x 7 stem, 3/4/6/3 bottleneck blocks)."""
    out, channels = [64 * 3 * 49, 64, 64], 64
    for blocks, width in ((3, 64), (4, 128), (6, 256), (3, 512)):
        for b in range(blocks):
            out += [width * channels, width, width, 9 * width * width, width, width,
                    4 * width * width, 4 * width, 4 * width]
            if b == 0:
                out += [4 * width * channels, 4 * width, 4 * width]
            channels = 4 * width
    return out + [channels * classes, classes]


def _numels(case):
    """Elements of a replica's tensors."""
    P, n = case["P"], case["n"]
    if n == 0:
        return [P]
    if (P, n) == (sum(_r50(100)), len(_r50(100))):
        return _r50(100)
    rng = random.Random(P * 1000 + n)
    cuts = sorted(int(P * rng.random() ** 3) for _ in range(n - 1))
    return [b - a for a, b in zip([0] + cuts, cuts + [P])]


def _gradient_inputs(case, gen):
    """Gradients of norms around max_norm (`long`: above), one value in 100 ten times as
    large; a replica's tensors lie in one row, each from a 16-byte boundary on."""
    W, dt = case["W"], _DT[case["dt"]]
    numels = _numels(case)
    starts, at = [], 0
    for n in numels:
        starts.append(at)
        at += _up(n, 8)
    ld = max(8, at)
    grads = torch.zeros((W, ld), dtype=dt, device="cuda")
    lo = 2.0 if case.get("long", False) else 0.4
    size = lo * torch.exp(torch.rand(W, generator=gen, device="cuda") * math.log(4.0))
    if case["mean"]:
        size = size.mean().expand(W) * W ** 0.5  # the mean of independent rows is shorter
    for i in range(W):
        v = torch.randn(ld, generator=gen, device="cuda")
        v = torch.where(torch.rand(ld, generator=gen, device="cuda") < 0.01, 10 * v, v)
        grads[i] = v * (size[i] / math.sqrt(2 * max(1, case["P"])))
    gap = torch.ones(ld, dtype=torch.bool)
    for s, n in zip(starts, numels):
        gap[s:s + n] = False
    if bool(gap.any()):
        grads[:, gap.cuda()] = 0
    return {"grads": grads, "ld": ld, "numels": numels, "starts": starts,
            "norm": torch.empty(1 if case["mean"] else W, device="cuda")}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] in ("score", "train"):
        st = _loss_inputs(case, gen)
    else:
        st = _gradient_inputs(case, gen)
    st["case"] = dict(case)
    if own:
        _own_prepare(st)
    return st


def run(state):
    return (_own if own else _plain)(state)


# ---- the calls of the framework -----------------------------------------------------

def _own_prepare(st):
    """What a program keeps from step to step: workspaces, and the plan of its tensors."""
    c = st["case"]
    if c["op"] in ("score", "train"):
        from paper_2607_21224_amd import q8
        need = q8.cpdp_q8_xent_workspace(c["T"], c["V"], c["K"])
        if c["op"] == "train":
            need = max(need, q8.cpdp_q8_xent_bwd_workspace(c["T"], c["V"], c["K"], _DT[c["dx"]],
                                                           _DT[c["dw"]]))
    else:
        from paper_2607_21224_amd import cpdp
        W, n = c["W"], c["n"]
        if n == 0:
            need = cpdp.cpdp_grad_norm_workspace(W, c["P"])
        else:
            rows = lambda t: [t[i, s:s + e] for i in range(W)  # noqa: E731
                              for s, e in zip(st["starts"], st["numels"])]
            st["params"] = torch.empty_like(st["grads"])
            st["mom"] = torch.empty_like(st["grads"])
            size = cpdp.cpdp_plan_bytes(W, n)
            st["table"] = torch.empty(size, dtype=torch.uint8, device="cuda")
            plan = st["plan"] = cpdp.cpdp_plan()
            plan.table = st["table"].data_ptr()
            cpdp.cpdp_plan_build(plan, size, W, n, st["numels"], rows(st["params"]),
                                 rows(st["mom"]), None, rows(st["grads"]), None, None)
            need = cpdp.cpdp_grad_norm_plan_workspace(plan)
    st["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")


def _own(st):
    c = st["case"]
    if c["op"] in ("score", "train"):
        from paper_2607_21224_amd import q8
        held = st["x"], st["xs"], st["w"], st["ws"], st["target"]
        q8.cpdp_q8_xent(*held, st["loss"], st["lse"], workspace=st["workspace"])
        if c["op"] == "train":
            q8.cpdp_q8_xent_bwd(*held, st["lse"], st["g"], st["dx"], st["dw"],
                                workspace=st["workspace"])
            return {k: st[k] for k in ("loss", "lse", "dx", "dw")}
        return {k: st[k] for k in ("loss", "lse")}
    from paper_2607_21224_amd import cpdp
    flags = cpdp.CPDP_NORM_MEAN if c["mean"] else 0
    if c["op"] == "norm":
        if c["n"]:
            cpdp.cpdp_grad_norm_plan(st["plan"], st["norm"], st["workspace"], flags=flags)
        else:
            cpdp.cpdp_grad_norm(st["grads"], c["W"], c["P"], st["ld"], st["norm"],
                                st["workspace"], c["dt"], flags=flags)
        return {"norm": st["norm"]}
    if c["n"]:
        cpdp.cpdp_clip_grads_plan(st["plan"], _MAX_NORM, st["norm"], st["workspace"],
                                  flags=flags)
    else:
        cpdp.cpdp_clip_grads(st["grads"], c["W"], c["P"], st["ld"], _MAX_NORM, st["norm"],
                             st["workspace"], c["dt"], flags=flags)
    return {"norm": st["norm"], "grads": st["grads"]}


# ---- the plain forms ------------------------------------------------------------------

def _plain(st):
    return _plain_loss(st) if st["case"]["op"] in ("score", "train") else _plain_clip(st)


def _plain_loss(st):
    c = st["case"]
    x = st["x"].float() * st["xs"][:, None]
    w = st["w"].float() * st["ws"][:, None]
    z = x @ w.t()
    top = z.amax(1)
    e = torch.exp(z - top[:, None])
    total = e.sum(1)
    lse = top + torch.log(total)
    counts = st["target"] >= 0
    at = st["target"].clamp_min(0)[:, None]
    loss = torch.where(counts, lse - z.gather(1, at)[:, 0], 0.0)
    out = {"loss": loss, "lse": lse}
    if c["op"] == "train":
        d = e / total[:, None]
        d.scatter_add_(1, at, torch.full_like(d[:, :1], -1.0))
        d = d * torch.where(counts, st["g"], 0.0)[:, None]
        out["dx"] = (d @ w).to(_DT[c["dx"]])
        out["dw"] = (d.t() @ x).to(_DT[c["dw"]])
    return out


def _plain_clip(st):
    c, g = st["case"], st["grads"]
    f = g.float()
    if c["mean"]:
        f = f.mean(0, keepdim=True)
    norm = torch.sqrt((f * f).sum(1))
    if c["op"] == "norm":
        return {"norm": norm}
    scale = torch.clamp(_MAX_NORM / (norm + 1e-6), max=1.0)
    g.copy_(g.float() * scale[:, None])
    return {"norm": norm, "grads": g}


# ---- the definitions in 64 bits ---------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    up = lambda t: t.to(torch.float64)  # noqa: E731
    if case["op"] in ("norm", "clip"):
        g = st["grads"]
        if case["mean"]:
            m = torch.zeros(st["ld"], dtype=torch.float64, device="cuda")
            for row in g:
                m += up(row)
            norm = torch.linalg.vector_norm(m / case["W"]).reshape(1)
        else:
            norm = torch.stack([torch.linalg.vector_norm(up(row)) for row in g])
        if case["op"] == "norm":
            return {"norm": norm}
        scale = torch.minimum(_MAX_NORM / (norm + 1e-6), torch.ones_like(norm))
        return {"norm": norm, "grads": up(g) * scale.unsqueeze(1)}
    T, V, K = case["T"], case["V"], case["K"]
    w = up(st["w"])
    ws, xs, target = up(st["ws"]), up(st["xs"]), st["target"]
    loss, lse = (torch.empty(T, dtype=torch.float64, device="cuda") for _ in range(2))
    train = case["op"] == "train"
    if train:
        dx = torch.empty((T, K), dtype=torch.float64, device="cuda")
        dw = torch.zeros((V, K), dtype=torch.float64, device="cuda")
    for t0 in range(0, T, 1024):
        s = slice(t0, min(T, t0 + 1024))
        x = up(st["x"][s]) * xs[s].unsqueeze(1)
        z = torch.mm(x, w.t()) * ws
        lse[s] = torch.logsumexp(z, 1)
        for_it = (target[s] >= 0).nonzero().flatten()
        hit = target[s][for_it]
        loss[s] = 0
        loss[t0 + for_it] = lse[t0 + for_it] - z[for_it, hit]
        if train:
            p = torch.exp(z - lse[s].unsqueeze(1))
            p[for_it, hit] -= 1
            p *= up(st["g"][s]).unsqueeze(1)
            p[target[s] < 0] = 0
            dx[s] = torch.mm(p * ws, w)
            dw += torch.mm(p.t(), x)
    out = {"loss": loss, "lse": lse}
    if train:
        out.update(dx=dx, dw=dw)
    return out
