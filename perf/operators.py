"""The operators of a residual student network at the sizes they are used at, in plain form and through the library.

Three operators, each forward and backward, over rows (vertices or tokens) of 32- and 16-bit elements:
  linear   Y = rho R + act(X W + 1 bias^T), and its gradients
  norm     X' = X + scale * gate * N_post(U), H = N_pre(X'): the norms around a block, with the block's gate and residual
           scale, and their gradients
  distill  loss and gradient of logits against a teacher's k largest logits per row, mixed with the labels' loss

Where `own` is false the operators are computed from elementary torch operations in 32 bits, rounded once at the end;
where it is true, by the library's calls.
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_EPS = 1e-5

_LIN = dict(op="linear", bias=True, residual=True, rho=1.0, keep=False)
_NORM = dict(op="norm", kind="rms", gate="full", post=True)
_KD = dict(op="distill", temperature=2.0, labelled=0.5, w_teacher=0.7, w_label=0.3)


def listed():
    return [
        # Answering for a single row: the product is one pass over the weights, and launches.
        dict(_LIN, name="linear_f32_one_row", pass_="forward", type="f32", n=1, k=1024, m=4096, act="silu"),
        # Sixteen rows at once (a small batch in serving): still one pass over 33 MB of weights.
        dict(_LIN, name="linear_bf16_sixteen_rows", pass_="forward", type="bf16", n=16, k=4096, m=4096, act="gelu"),
        # The features of a graph of 232,965 vertices (602 of them) into hidden width 128: tall, narrow, bound by memory
        # and by the 32-bit matrix rate alike.
        dict(_LIN, name="linear_f32_features", pass_="forward", type="f32", n=232_965, k=602, m=128, act="relu",
             residual=False),
        # The wide product of a training step, the pre-activation kept for backward: bound by the matrix units.
        dict(_LIN, name="linear_bf16_wide", pass_="forward", type="bf16", n=16_384, k=4096, m=4096, act="gelu", keep=True),
        # Backward of a block's first product: two products and an elementwise pass.
        dict(_LIN, name="linear_f16_backward", pass_="backward", type="f16", n=8192, k=1024, m=4096, act="silu"),
        # Nothing aligned: odd row count, rows of 602 and of 1001 16-bit elements, a scaled residual.
        dict(_LIN, name="linear_bf16_backward_ragged", pass_="backward", type="bf16", n=4099, k=602, m=1001, act="gelu",
             rho=0.5),
        # One row through the norms between two blocks: latency and nothing else.
        dict(_NORM, name="norm_bf16_one_row", pass_="forward", type="bf16", n=1, f=4096),
        # All vertices of that graph at hidden width 128, layer norm with its biases.
        dict(_NORM, name="norm_f32_vertices", pass_="forward", type="f32", n=232_965, f=128, kind="layer"),
        # A training step's backward: eight matrices of 134 MB, and sums over all rows for four vectors.
        dict(_NORM, name="norm_bf16_backward", pass_="backward", type="bf16", n=16_384, f=4096),
        # Odd width, one gate per row (broadcast, so that its gradient is a sum over the row), layer norm.
        dict(_NORM, name="norm_f16_backward_ragged", pass_="backward", type="f16", n=8195, f=301, kind="layer", gate="row"),
        # Vertex classes: short rows of 41, the teacher's eight largest, half of the vertices labelled.
        dict(_KD, name="distill_f32_classes", type="f32", n=232_965, c=41, k=8),
        # A vocabulary: rows of 200 KB, read once and written once, 64 entries of the teacher in each.
        dict(_KD, name="distill_bf16_vocabulary", type="bf16", n=4096, c=100_000, k=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Half of the sizes are multiples of 64 (of 8 where small), as models have them; the others are whatever comes."""
    s = _log(rng, lo, hi)
    if rng.random() < 0.5:
        unit = 64 if s >= 64 else 8
        s = max(unit, s // unit * unit)
    return max(lo, min(hi, s))


def draw(rng):
    op = rng.choice(["linear", "linear", "norm", "distill"])
    case = dict(type=rng.choice(["f32", "bf16", "f16"]))
    if op == "linear":
        k, m = _size(rng, 16, 4096), _size(rng, 16, 4096)
        back = rng.random() < 0.5
        most = 2.5e11 / (2.0 * k * m * (2 if back else 1)) / (4 if case["type"] == "f32" else 1)
        n = max(1, min(_log(rng, 1, 262_144), int(most), int(4e8 / max(k, m))))
        case.update(_LIN, pass_="backward" if back else "forward", n=n, k=k, m=m, act=rng.choice(["none", "relu", "gelu", "silu"]),
                    bias=rng.random() < 0.8, residual=rng.random() < 0.6, rho=rng.choice([1.0, 1.0, 0.5]),
                    keep=rng.random() < 0.5)
    elif op == "norm":
        f = _size(rng, 16, 8192)
        n = max(1, min(_log(rng, 1, 262_144), int(6e7 / f)))
        case.update(_NORM, pass_=rng.choice(["forward", "backward"]), n=n, f=f, kind=rng.choice(["rms", "layer"]),
                    gate=rng.choice(["none", "row", "full", "full"]), post=rng.random() < 0.8)
    else:
        c = _size(rng, 8, 131_072)
        n = max(1, min(_log(rng, 1, 262_144), int(2e8 / c)))
        case.update(_KD, n=n, c=c, k=min(c, _log(rng, 1, 64)), temperature=rng.choice([1.0, 2.0, 4.0]),
                    labelled=rng.choice([0.0, 0.5, 1.0]))
    return case


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _normal(gen, shape, type_, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(_TYPES[type_])


def _empty(shape, type_="f32"):
    return torch.empty(shape, dtype=_TYPES[type_], device="cuda")


def _prepare_linear(c, gen):
    n, k, m, t = c["n"], c["k"], c["m"], c["type"]
    s = dict(X=_normal(gen, (n, k), t), W=_normal(gen, (k, m), t, k ** -0.5))
    if c["pass_"] == "forward":
        s["bias"] = _normal(gen, (m,), "f32", 0.1) if c["bias"] else None
        s["R"] = _normal(gen, (n, m), t) if c["residual"] else None
        s["Y"] = _empty((n, m), t)
        s["Z"] = _empty((n, m), t) if c["keep"] else None
    else:
        s["Z"] = _normal(gen, (n, m), t)                       # what the forward pass kept
        s["dY"] = _normal(gen, (n, m), t)
        s["dZ"] = _empty((n, m), t)                            # workspace
        s["dX"], s["dW"] = _empty((n, k), t), _empty((k, m), t)
        s["dbias"] = _empty((m,)) if c["bias"] else None
        s["dR"] = _empty((n, m), t) if c["residual"] and c["rho"] != 1.0 else None
    return s


def _prepare_norm(c, gen):
    n, f, t = c["n"], c["f"], c["type"]
    layer = c["kind"] == "layer"

    def weight():
        return 1.0 + 0.1 * torch.randn(f, generator=gen, device="cuda")

    s = dict(U=_normal(gen, (n, f), t, 2.0), scale=0.2 * weight(), w_pre=weight())
    s["A"] = None if c["gate"] == "none" else _normal(gen, (n, f if c["gate"] == "full" else 1), t)
    s["w_post"] = weight() if c["post"] else None
    s["b_post"] = _normal(gen, (f,), "f32", 0.1) if layer and c["post"] else None
    s["b_pre"] = _normal(gen, (f,), "f32", 0.1) if layer else None
    s["stats"] = _empty((n, 4))
    if c["pass_"] == "forward":
        s["X"] = _normal(gen, (n, f), t)
        s["Xout"], s["H"] = _empty((n, f), t), _empty((n, f), t)
        return s
    s["Xout"] = _normal(gen, (n, f), t, 1.2)                   # what the forward pass wrote, and the statistics that it kept
    for at, rows in ((0, s["U"]), (2, s["Xout"])):
        x = rows.float()
        mean = x.mean(1) if layer else torch.zeros(n, device="cuda")
        s["stats"][:, at] = mean
        s["stats"][:, at + 1] = ((x - mean[:, None]).square().mean(1) + _EPS).rsqrt()
    s["dXout"], s["dH"] = _normal(gen, (n, f), t), _normal(gen, (n, f), t)
    s["dX"], s["dU"] = _empty((n, f), t), _empty((n, f), t)
    s["dA"] = None if s["A"] is None else torch.empty_like(s["A"])
    s["dscale"], s["dw_pre"] = _empty((f,)), _empty((f,))
    s["dw_post"] = _empty((f,)) if c["post"] else None
    s["db_post"] = _empty((f,)) if s["b_post"] is not None else None
    s["db_pre"] = _empty((f,)) if s["b_pre"] is not None else None
    return s


def _prepare_distill(c, gen):
    n, cols, k = c["n"], c["c"], c["k"]
    Z = _normal(gen, (n, cols), c["type"], 2.0)
    # The teacher agrees with the student in part: its largest logits are largest among the student's, moved by noise.
    top = torch.empty(n, k, dtype=torch.int32, device="cuda")
    t = torch.empty(n, k, dtype=_TYPES[c["type"]], device="cuda")
    step = max(1, (1 << 27) // cols)
    for at in range(0, n, step):
        z = Z[at:at + step].float()
        v, i = (0.7 * z + torch.randn(z.shape, generator=gen, device="cuda")).topk(k, dim=1)
        top[at:at + step], t[at:at + step] = i.int(), (1.5 * v).to(t.dtype)
    # a short list here and there (absent entries have a negative index), and rows that the teacher never saw
    top[torch.rand(n, k, generator=gen, device="cuda") < 0.05] = -1
    top[torch.rand(n, generator=gen, device="cuda") < 0.05] = -1
    y = torch.randint(cols, (n,), generator=gen, device="cuda", dtype=torch.int32)
    y[torch.rand(n, generator=gen, device="cuda") >= c["labelled"]] = -1
    return dict(Z=Z, top=top, t=t, labels=y, loss=_empty((1,)), G=torch.empty_like(Z))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    make = {"linear": _prepare_linear, "norm": _prepare_norm, "distill": _prepare_distill}[case["op"]]
    return dict(make(case, gen), case=case)


# ---- plain forms ----------------------------------------------------------------------------------------------------
def _f(t):
    return None if t is None else t.float()


def _act(z, act):
    if act == "none":
        return z
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))


def _slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "silu":
        sig = 1 / (1 + torch.exp(-z))
        return sig * (1 + z * (1 - sig))
    return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)


def _plain_linear(c, s):
    t = _TYPES[c["type"]]
    X, W = _f(s["X"]), _f(s["W"])
    if c["pass_"] == "forward":
        z = X @ W
        if s["bias"] is not None:
            z = z + s["bias"]
        y = _act(z, c["act"])
        if s["R"] is not None:
            y = y + c["rho"] * _f(s["R"])
        return {"Y": y.to(t), "Z": z.to(t)} if c["keep"] else {"Y": y.to(t)}
    dY = _f(s["dY"])
    dZ = dY if c["act"] == "none" else dY * _slope(_f(s["Z"]), c["act"])
    out = {"dX": (dZ @ W.t()).to(t), "dW": (X.t() @ dZ).to(t)}
    if s["dbias"] is not None:
        out["dbias"] = dZ.sum(0)
    if s["dR"] is not None:
        out["dR"] = (c["rho"] * dY).to(t)
    return out


def _unit(x, layer):
    """x normalised by its row, and the rows' statistics."""
    mean = x.mean(1, keepdim=True) if layer else torch.zeros_like(x[:, :1])
    rstd = ((x - mean).square().mean(1, keepdim=True) + _EPS).rsqrt()
    return (x - mean) * rstd, mean, rstd


def _unit_gradient(g, unit, rstd, layer):
    along = (g * unit).mean(1, keepdim=True)
    return rstd * (g - unit * along - (g.mean(1, keepdim=True) if layer else 0))


def _plain_norm(c, s):
    t, layer = _TYPES[c["type"]], c["kind"] == "layer"
    U = _f(s["U"])
    gate = 1.0 if s["A"] is None else 1 / (1 + torch.exp(-_f(s["A"])))
    if c["pass_"] == "forward":
        stats = torch.zeros_like(s["stats"])
        v = U
        if c["post"]:
            unit, mean, rstd = _unit(U, layer)
            v = unit * s["w_post"]
            if layer:
                v = v + s["b_post"]
            stats[:, 0:1], stats[:, 1:2] = mean, rstd
        x = _f(s["X"]) + s["scale"] * (gate * v)
        unit, mean, rstd = _unit(x, layer)
        h = unit * s["w_pre"]
        if layer:
            h = h + s["b_pre"]
        stats[:, 2:3], stats[:, 3:4] = mean, rstd
        return {"Xout": x.to(t), "H": h.to(t), "stats": stats}
    mean, rstd, xmean, xrstd = s["stats"].split(1, dim=1)
    out = {}
    dH = _f(s["dH"])
    xunit = (_f(s["Xout"]) - xmean) * xrstd
    out["dw_pre"] = (dH * xunit).sum(0)
    if layer:
        out["db_pre"] = dH.sum(0)
    dx = _f(s["dXout"]) + _unit_gradient(dH * s["w_pre"], xunit, xrstd, layer)
    out["dX"] = dx.to(t)
    unit = (U - mean) * rstd if c["post"] else U
    v = unit * s["w_post"] if c["post"] else U
    if layer and c["post"]:
        v = v + s["b_post"]
    out["dscale"] = (dx * gate * v).sum(0)
    if s["A"] is not None:
        dA = dx * s["scale"] * v * gate * (1 - gate)
        out["dA"] = (dA if c["gate"] == "full" else dA.sum(1, keepdim=True)).to(t)
    dv = dx * s["scale"] * gate
    if c["post"]:
        out["dw_post"] = (dv * unit).sum(0)
        if layer:
            out["db_post"] = dv.sum(0)
        dv = _unit_gradient(dv * s["w_post"], unit, rstd, layer)
    out["dU"] = dv.to(t)
    return out


def _plain_softmax(z):
    """softmax and log-softmax along rows; a row of -inf alone gives zeros."""
    high = z.max(1, keepdim=True).values
    high = torch.where(high == -math.inf, torch.zeros_like(high), high)
    e = torch.exp(z - high)
    total = e.sum(1, keepdim=True)
    return torch.where(total > 0, e / total, torch.zeros_like(e)), z - high - torch.log(total)


def _plain_distill(c, s):
    n, T = c["n"], c["temperature"]
    z = _f(s["Z"])
    q, logq = _plain_softmax(z / T)
    there = s["top"] >= 0
    at = s["top"].clamp(min=0).long()
    p, logp = _plain_softmax(torch.where(there, _f(s["t"]) / T, torch.full_like(s["t"], -math.inf, dtype=torch.float32)))
    kl = torch.where(p > 0, p * (logp - logq.gather(1, at)), torch.zeros_like(p)).sum()
    G = q * there.any(1, keepdim=True)
    G = (c["w_teacher"] * T) * G.scatter_add(1, at, -p)
    del q, logq
    soft, logsoft = _plain_softmax(z)
    known = (s["labels"] >= 0)[:, None]
    y = s["labels"].clamp(min=0).long()[:, None]
    nll = -torch.where(known, logsoft.gather(1, y), torch.zeros_like(logsoft[:, :1])).sum()
    G += c["w_label"] * (soft.scatter_add(1, y, torch.full_like(soft[:, :1], -1.0)) * known)
    return {"loss": ((c["w_teacher"] * T * T) * kl + c["w_label"] * nll).reshape(1) / n, "G": (G / n).to(_TYPES[c["type"]])}


# ---- the library's calls --------------------------------------------------------------------------------------------
def _own_linear(c, s):
    import paper_2005_03300_amd as g
    act = {"none": g.ACT_NONE, "relu": g.ACT_RELU, "gelu": g.ACT_GELU, "silu": g.ACT_SILU}[c["act"]]
    if c["pass_"] == "forward":
        g.gcn_linear_forward(s["X"], s["W"], s["Y"], bias=s["bias"], act=act, R=s["R"], rho=c["rho"], Z=s["Z"])
        return {"Y": s["Y"], "Z": s["Z"]} if c["keep"] else {"Y": s["Y"]}
    g.gcn_linear_backward(s["X"], s["W"], s["Z"], s["dY"], s["dZ"], dX=s["dX"], dW=s["dW"], dbias=s["dbias"], act=act,
                          dR=s["dR"], rho=c["rho"])
    return {k: s[k] for k in ("dX", "dW", "dbias", "dR") if s[k] is not None}


def _own_norm(c, s):
    import paper_2005_03300_amd as g
    kind = g.NORM_LAYER if c["kind"] == "layer" else g.NORM_RMS
    if c["pass_"] == "forward":
        g.gcn_block_norm_forward(s["X"], s["U"], s["Xout"], s["H"], w_pre=s["w_pre"], b_pre=s["b_pre"], A=s["A"],
                                 scale=s["scale"], w_post=s["w_post"], b_post=s["b_post"], stats=s["stats"], kind=kind, eps=_EPS)
        return {k: s[k] for k in ("Xout", "H", "stats")}
    g.gcn_block_norm_backward(s["U"], s["Xout"], s["stats"], s["dXout"], s["dH"], s["dX"], s["dU"], w_pre=s["w_pre"],
                              A=s["A"], dA=s["dA"], scale=s["scale"], w_post=s["w_post"], b_post=s["b_post"],
                              dscale=s["dscale"], dw_post=s["dw_post"], db_post=s["db_post"], dw_pre=s["dw_pre"],
                              db_pre=s["db_pre"], kind=kind)
    return {k: s[k] for k in ("dX", "dU", "dA", "dscale", "dw_post", "db_post", "dw_pre", "db_pre") if s[k] is not None}


def _own_distill(c, s):
    import paper_2005_03300_amd as g
    g.gcn_distill(s["Z"], s["top"], s["t"], s["loss"], s["G"], labels=s["labels"], temperature=c["temperature"],
                  w_teacher=c["w_teacher"], w_label=c["w_label"])
    return {"loss": s["loss"], "G": s["G"]}


_PLAIN = {"linear": _plain_linear, "norm": _plain_norm, "distill": _plain_distill}
_OWN = {"linear": _own_linear, "norm": _own_norm, "distill": _own_distill}


def run(state):
    c = state["case"]
    return (_OWN if own else _PLAIN)[c["op"]](c, state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    c, e = case, _BYTES[case["type"]]
    if c["op"] == "linear":
        n, k, m = c["n"], c["k"], c["m"]
        if c["pass_"] == "forward":
            mats = n * k + k * m + n * m * (1 + bool(c["residual"]) + bool(c["keep"]))
            return {"bytes": e * mats + 4 * m * bool(c["bias"]), "flops": 2 * n * k * m}
        scaled = c["residual"] and c["rho"] != 1.0
        mats = 2 * n * k + 2 * k * m + n * m * (1 + (c["act"] != "none") + scaled)
        return {"bytes": e * mats + 4 * m * bool(c["bias"]), "flops": 4 * n * k * m}
    if c["op"] == "norm":
        n, f = c["n"], c["f"]
        gate = {"none": 0, "row": n, "full": n * f}[c["gate"]]
        vectors = 1 + (1 + (c["kind"] == "layer")) * (1 + bool(c["post"]))
        if c["pass_"] == "forward":
            return {"bytes": e * (4 * n * f + gate) + 4 * (vectors * f + 4 * n), "flops": 16 * n * f}
        return {"bytes": e * (6 * n * f + 2 * gate) + 4 * (2 * vectors * f + 4 * n), "flops": 32 * n * f}
    n, cols, k = c["n"], c["c"], c["k"]
    return {"bytes": 2 * e * n * cols + n * k * (4 + e) + 4 * n, "flops": 10 * n * cols}


# ---- from the definitions, in 64 bits -------------------------------------------------------------------------------
def _d(t):
    return None if t is None else t.double()


def _exact_linear(c, s):
    f = {"none": lambda z: z, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[c["act"]]
    X, W = _d(s["X"]), _d(s["W"])
    if c["pass_"] == "forward":
        z = X @ W if s["bias"] is None else torch.addmm(s["bias"].double(), X, W)
        y = f(z) if s["R"] is None else torch.add(f(z), s["R"].double(), alpha=c["rho"])
        return {"Y": y, "Z": z} if c["keep"] else {"Y": y}
    z = _d(s["Z"]).requires_grad_()
    dZ, = torch.autograd.grad(f(z), z, _d(s["dY"]))
    out = {"dX": dZ @ W.t(), "dW": X.t() @ dZ, "dbias": dZ.sum(0), "dR": c["rho"] * _d(s["dY"])}
    return {k: v for k, v in out.items() if s[k] is not None}


def _exact_norm(c, s):
    layer = c["kind"] == "layer"

    def norm(x, w, b, mean=None, rstd=None):
        mean = (x.mean(1, keepdim=True) if layer else 0 * x[:, :1]) if mean is None else mean
        x = x - mean
        rstd = 1 / torch.sqrt((x * x).mean(1, keepdim=True) + _EPS) if rstd is None else rstd
        y = x * rstd * w
        return (y if b is None else y + b), mean, rstd

    U, A = _d(s["U"]), _d(s["A"])
    scale, w_post, b_post, w_pre, b_pre = (_d(s[k]) for k in ("scale", "w_post", "b_post", "w_pre", "b_pre"))
    if c["pass_"] == "forward":
        v, mean, rstd = norm(U, w_post, b_post) if c["post"] else (U, 0 * U[:, :1], 0 * U[:, :1])
        x = _d(s["X"]) + scale * v * (1.0 if A is None else torch.sigmoid(A))
        h, xmean, xrstd = norm(x, w_pre, b_pre)
        return {"Xout": x, "H": h, "stats": torch.cat([mean, rstd, xmean, xrstd], 1)}
    # The gradient by differentiation. The statistics that the forward pass kept are those of the rows up to roundings of 32
    # bits, so they are taken anew; X' is given, and what comes before it differentiated apart from what comes after.
    leaf = {k: v.requires_grad_() for k, v in dict(U=U, A=A, dscale=scale, dw_post=w_post, db_post=b_post).items() if v is not None}
    xo = _d(s["Xout"]).requires_grad_()
    after = {k: v.requires_grad_() for k, v in dict(dw_pre=w_pre, db_pre=b_pre).items() if v is not None}
    h = norm(xo, w_pre, b_pre)[0]
    got = torch.autograd.grad(h, [xo, *after.values()], _d(s["dH"]))
    out = dict(zip(after, got[1:]))
    out["dX"] = got[0] + _d(s["dXout"])
    v = norm(U, w_post, b_post)[0] if c["post"] else U
    y = scale * v * (1.0 if A is None else torch.sigmoid(A))
    out.update(zip(({"U": "dU", "A": "dA"}.get(k, k) for k in leaf), torch.autograd.grad(y, list(leaf.values()), out["dX"])))
    return out


def _exact_distill(c, s):
    n, T = c["n"], c["temperature"]
    loss, G = 0.0, torch.empty(s["Z"].shape, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 26) // c["c"])
    for at in range(0, n, step):
        z = s["Z"][at:at + step].double().requires_grad_()
        top, y = s["top"][at:at + step], s["labels"][at:at + step].long()
        t = s["t"][at:at + step].double().div(T).masked_fill(top < 0, -math.inf)
        seen = (top >= 0).any(1)
        p = torch.softmax(torch.where(seen[:, None], t, torch.zeros_like(t)), 1) * seen[:, None]
        logq = torch.log_softmax(z / T, 1).gather(1, top.clamp(min=0).long())
        part = (c["w_teacher"] * T * T) * (torch.special.xlogy(p, p) - p * logq).sum()
        part = part + c["w_label"] * torch.nn.functional.cross_entropy(z, y, ignore_index=-1, reduction="sum")
        G[at:at + step], = torch.autograd.grad(part / n, z)
        loss = loss + part.detach() / n
    return {"loss": loss.reshape(1), "G": G}


def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "norm": _exact_norm, "distill": _exact_distill}[case["op"]](case, s)
