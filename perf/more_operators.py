"""Gated blocks of a residual student network, the 8-bit checkpoints that they are trained with and the 4-bit weights that they
answer with, at the sizes they are used at, in plain form and through the library.

Three operators over rows (vertices or tokens) of 32- and 16-bit elements:
  gated       Z = X W + 1 bias^T with W: k x 2 m, H = act(Z[:, :m]) * Z[:, m:], and its gradients, from what the forward pass kept
              or from checkpoints of it
  checkpoint  a matrix of activations held in 8 bits: each 64 neighbours of a row have a scale s, the smallest bf16 number with
              127 s >= |x| for all of them, and x is held as the whole number c nearest to x / s (ties to even); it stands for s c,
              rounded to the element type.  Stored and restored; and the backward pass of a linear layer, Y = rho R + act(X W + 1 bias^T),
              from checkpoints of X and of act's argument
  linear4     Y = rho R + act(X W + 1 bias^T), or the gated block, with W held in 4 bits: each `group` neighbours of a column have a
              scale s, the smallest bf16 number with 6 s >= |w|, and w is held as the nearest of +-s {0, 1/2, 1, 3/2, 2, 3, 4, 6} (ties
              to the even code).  A code has the sign in bit 3 and the place in that list in bits 0 to 2; word (j, n) of the codes holds those of
              W[8 j .. 8 j + 7, n], the first in its lowest bits

Where `own` is false the operators are computed from elementary torch operations in 32 bits, rounded once at the end (the codes, which
lie next to borders, in 64); where it is true, by the library's calls.
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_GROUP = 64                                                        # of a checkpoint
_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)

_GATED = dict(op="gated", act="silu", bias=True, keep=False, held8=False)
_CHECK = dict(op="checkpoint", act="gelu", bias=True, rho=1.0)
_LIN4 = dict(op="linear4", gated=False, act="none", bias=True, residual=False, rho=1.0)


def listed():
    return [
        # Answering for a single row: both projections are one pass over 134 MB of weights.
        dict(_GATED, name="gated_bf16_one_row", pass_="forward", type="bf16", n=1, k=4096, m=8192),
        # A training step's forward pass, the argument kept for backward: bound by the matrix units.
        dict(_GATED, name="gated_bf16_wide", pass_="forward", type="bf16", n=8192, k=2048, m=8192, keep=True),
        # All vertices of a graph of 232,965 at hidden width 128: tall and narrow, bound by memory and by the 32-bit products.
        dict(_GATED, name="gated_f32_vertices", pass_="forward", type="f32", n=232_965, k=128, m=256, act="gelu"),
        # The same step's backward pass: an elementwise pass, which also gives H again for the next layer's weights, and two products.
        dict(_GATED, name="gated_f16_backward", pass_="backward", type="f16", n=8192, k=1024, m=4096),
        # Backward from checkpoints with nothing aligned: odd row count, rows of 602 and of 1001 elements, whose last groups are short.
        dict(_GATED, name="gated_bf16_backward_ragged", pass_="backward", type="bf16", n=4099, k=602, m=1001, act="gelu", held8=True),
        # The features of that graph (602 for each vertex) stored in 8 bits and restored.
        dict(_CHECK, name="checkpoint_bf16_features", pass_="restore", type="bf16", n=232_965, k=602),
        # A training step's backward pass of a wide layer from checkpoints: two products of 550 GFLOP.
        dict(_CHECK, name="checkpoint_bf16_backward", pass_="backward", type="bf16", n=16_384, k=4096, m=4096),
        # The same of all vertices at width 128, in 32 bits, where a checkpoint is a quarter of the activations.
        dict(_CHECK, name="checkpoint_f32_backward_vertices", pass_="backward", type="f32", n=232_965, k=128, m=256, act="relu"),
        # Answering for one row from 4-bit weights: the smallest call, where the launch counts.
        dict(_LIN4, name="linear4_bf16_one_row", pass_="forward", type="bf16", n=1, k=4096, m=4096, group=64, act="silu"),
        # A batch of sixteen through a gated block: one pass over 117 MB of codes.
        dict(_LIN4, name="linear4_f16_gated_sixteen_rows", pass_="forward", type="f16", n=16, k=8192, m=14_336, group=128, gated=True, act="silu"),
        # Many rows at once (a long request, or all of a small graph) with the finest groups: bound by the matrix units.
        dict(_LIN4, name="linear4_bf16_many_rows", pass_="forward", type="bf16", n=2048, k=4096, m=4096, group=32, residual=True, rho=0.5),
        # Weights laid out in 4 bits from their 32-bit copies and read back; a height that ends inside a group and a word.
        dict(_LIN4, name="linear4_f32_restore", pass_="restore", type="f32", n=0, k=4099, m=4096, group=64),
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
    op = rng.choice(["gated", "gated", "checkpoint", "linear4", "linear4"])
    case = dict(type=rng.choice(["f32", "bf16", "f16"]))
    k, m = _size(rng, 16, 4096), _size(rng, 16, 4096)
    act = rng.choice(["none", "relu", "gelu", "silu"])
    slow = 4 if case["type"] == "f32" else 1

    def rows(products, most=262_144):
        return max(1, min(_log(rng, 1, most), int(2.5e11 / (2.0 * k * m * products) / slow), int(4e8 / max(k, 2 * m))))

    if op == "gated":
        back = rng.random() < 0.5
        case.update(_GATED, pass_="backward" if back else "forward", n=rows(4 if back else 2), k=k, m=m, act=act,
                    bias=rng.random() < 0.8, keep=not back and rng.random() < 0.5, held8=back and rng.random() < 0.5)
    elif op == "checkpoint":
        if rng.random() < 0.3:
            case.update(_CHECK, pass_="restore", n=max(1, min(_log(rng, 1, 262_144), int(2e8 / k))), k=k)
        else:
            case.update(_CHECK, pass_="backward", n=rows(2), k=k, m=m, act=act, bias=rng.random() < 0.8, rho=rng.choice([1.0, 0.5]))
    else:
        case.update(_LIN4, group=rng.choice([32, 64, 128]), k=_size(rng, 16, 8192), m=_size(rng, 16, 8192))
        if rng.random() < 0.15:
            case.update(pass_="restore", n=0)
        else:
            gated = rng.random() < 0.4
            k, m = case["k"], case["m"]
            n = rows(2 if gated else 1) if rng.random() < 0.3 else _log(rng, 1, 64)
            case.update(pass_="forward", n=n, gated=gated, act=act, bias=rng.random() < 0.5, residual=rng.random() < 0.5,
                        rho=rng.choice([1.0, 0.5]))
    return case


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _normal(gen, shape, type_, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(_TYPES[type_])


def _empty(shape, type_="f32"):
    return torch.empty(shape, dtype=_TYPES[type_], device="cuda")


def _held(shape):
    """Room for a checkpoint of a matrix of that shape."""
    n, f = shape
    return torch.empty(n, f, dtype=torch.int8, device="cuda"), torch.empty(n, -(-f // _GROUP), dtype=torch.bfloat16, device="cuda")


def _held4(k, cols, group):
    return (torch.empty(-(-k // 8), cols, dtype=torch.int32, device="cuda"), torch.empty(-(-k // group), cols, dtype=torch.bfloat16, device="cuda"))


def _prepare_gated(c, gen):
    n, k, m, t = c["n"], c["k"], c["m"], c["type"]
    s = dict(X=_normal(gen, (n, k), t), W=_normal(gen, (k, 2 * m), t, k ** -0.5))
    if c["pass_"] == "forward":
        s["bias"] = _normal(gen, (2 * m,), "f32", 0.1) if c["bias"] else None
        s["H"] = _empty((n, m), t)
        s["Z"] = _empty((n, 2 * m), t) if c["keep"] else None
        return s
    s["Z"] = _normal(gen, (n, 2 * m), t)                           # what the forward pass kept
    if c["held8"]:
        s["X"], s["Z"] = _pack(s["X"]), _pack(s["Z"])
    s["dH"] = _normal(gen, (n, m), t)
    s["dZ"] = _empty((n, 2 * m), t)                                # workspace
    s["H"], s["dX"], s["dW"] = _empty((n, m), t), _empty((n, k), t), _empty((k, 2 * m), t)
    s["dbias"] = _empty((2 * m,)) if c["bias"] else None
    return s


def _prepare_checkpoint(c, gen):
    n, k, t = c["n"], c["k"], c["type"]
    X = _normal(gen, (n, k), t)
    if c["pass_"] == "restore":
        # columns of very different sizes, as features have them, and some rows that are small as a whole or zero
        X *= torch.exp(2 * torch.randn(k, generator=gen, device="cuda")).clamp(max=100).to(X.dtype)
        X *= (torch.rand(n, 1, generator=gen, device="cuda") * 8).floor().div(7).to(X.dtype)
        return dict(X=X, held=_held((n, k)), back=torch.empty_like(X))
    m = c["m"]
    s = dict(X=_pack(X), W=_normal(gen, (k, m), t, k ** -0.5), Z=_pack(_normal(gen, (n, m), t)), dY=_normal(gen, (n, m), t))
    s["dZ"] = _empty((n, m), t)                                    # workspace
    s["dX"], s["dW"] = _empty((n, k), t), _empty((k, m), t)
    s["dbias"] = _empty((m,)) if c["bias"] else None
    s["dR"] = _empty((n, m), t) if c["rho"] != 1.0 else None
    return s


def _prepare_linear4(c, gen):
    n, k, m, t, group = c["n"], c["k"], c["m"], c["type"], c["group"]
    cols = 2 * m if c["gated"] else m
    W = _normal(gen, (k, cols), t, k ** -0.5)
    if c["pass_"] == "restore":
        return dict(W=W, held=_held4(k, cols, group), back=torch.empty_like(W))
    s = dict(X=_normal(gen, (n, k), t), held=_pack4(W, group), Y=_empty((n, m), t))
    s["bias"] = _normal(gen, (cols,), "f32", 0.1) if c["bias"] else None
    s["R"] = _normal(gen, (n, m), t) if c["residual"] else None
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    make = {"gated": _prepare_gated, "checkpoint": _prepare_checkpoint, "linear4": _prepare_linear4}[case["op"]]
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
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0).float()
    if act == "silu":
        sig = 1 / (1 + torch.exp(-z))
        return sig * (1 + z * (1 - sig))
    return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)


def _scales(most, steps):
    """The smallest bf16 numbers s, 2^-126 at least, with steps * s >= most."""
    s = (most.float() / steps).to(torch.bfloat16).clamp(min=2.0 ** -126)
    return torch.where(steps * s.float() < most.float(), (s.view(torch.int16) + 1).view(torch.bfloat16), s)


def _grouped(x, size):
    """The rows of x in groups, the last one of zeros at its end."""
    n, f = x.shape
    out = x.new_zeros(n, -(-f // size), size)
    out.view(n, -1)[:, :f] = x
    return out


def _pack(x):
    f = x.shape[1]
    g = _grouped(x, _GROUP)
    s = _scales(g.abs().amax(2), 127.0)
    c = torch.round(g.double() / s.double()[:, :, None])
    return c.to(torch.int8).view(x.shape[0], -1)[:, :f].contiguous(), s


def _unpack(held, t):
    c, s = held
    return (c.float() * s.float().repeat_interleave(_GROUP, 1)[:, :c.shape[1]]).to(t)


def _pack4(w, group):
    k, cols = w.shape
    g = _grouped(w.t(), group)                                     # cols x groups x group
    s = _scales(g.abs().amax(2), 6.0)
    # Next to the borders between two places: products with a scale of eight bits, which are exact.  A border itself goes to the even place.
    border = torch.tensor((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0), device=w.device) * s.float()[:, :, None, None]
    a = g.abs().float()[:, :, :, None]
    up = torch.tensor((0, 1, 0, 1, 0, 1, 0), device=w.device, dtype=torch.bool)
    code = ((a > border) | ((a == border) & up)).sum(3, dtype=torch.int32)
    code += 8 * ((g < 0) & (code > 0))
    words = _grouped(code.view(cols, -1)[:, :k], 8)                # cols x words x 8
    words = (words << torch.arange(0, 32, 4, device=w.device, dtype=torch.int32)).sum(2, dtype=torch.int32)
    return words.t().contiguous(), s.t().contiguous()


def _unpack4(held, k, group):
    q, s = held
    code = (q[:, None, :] >> torch.arange(0, 32, 4, device=q.device, dtype=torch.int32)[None, :, None]) & 15
    code = code.reshape(-1, q.shape[1])[:k]
    size = torch.tensor(_LEVELS, device=q.device)[(code & 7).long()]
    return torch.where(code >= 8, -size, size) * s.float().repeat_interleave(group, 0)[:k]


def _seen(held, t):
    """What a pass has in hand: a matrix, or the one that a checkpoint stands for."""
    return _f(_unpack(held, t)) if isinstance(held, tuple) else _f(held)


def _plain_gated(c, s):
    t, m = _TYPES[c["type"]], c["m"]
    if c["pass_"] == "forward":
        z = _f(s["X"]) @ _f(s["W"])
        if s["bias"] is not None:
            z = z + s["bias"]
        h = (_act(z[:, :m], c["act"]) * z[:, m:]).to(t)
        return {"H": h, "Z": z.to(t)} if c["keep"] else {"H": h}
    X, Z, dH = _seen(s["X"], t), _seen(s["Z"], t), _f(s["dH"])
    zg, zu = Z[:, :m], Z[:, m:]
    a = _act(zg, c["act"])
    dZ = torch.cat([dH * zu * _slope(zg, c["act"]), dH * a], 1)
    out = {"H": (a * zu).to(t), "dX": (dZ @ _f(s["W"]).t()).to(t), "dW": (X.t() @ dZ).to(t)}
    if s["dbias"] is not None:
        out["dbias"] = dZ.sum(0)
    return out


def _plain_checkpoint(c, s):
    t = _TYPES[c["type"]]
    if c["pass_"] == "restore":
        held = _pack(s["X"])
        return {"X": _unpack(held, t), "scales": held[1]}
    dY = _f(s["dY"])
    dZ = dY if c["act"] == "none" else dY * _slope(_seen(s["Z"], t), c["act"])
    out = {"dX": (dZ @ _f(s["W"]).t()).to(t), "dW": (_seen(s["X"], t).t() @ dZ).to(t)}
    if s["dbias"] is not None:
        out["dbias"] = dZ.sum(0)
    if s["dR"] is not None:
        out["dR"] = (c["rho"] * dY).to(t)
    return out


def _plain_linear4(c, s):
    t, m = _TYPES[c["type"]], c["m"]
    if c["pass_"] == "restore":
        held = _pack4(s["W"], c["group"])
        return {"W": _unpack4(held, c["k"], c["group"]).to(t), "scales": held[1]}
    z = _f(s["X"]) @ _unpack4(s["held"], c["k"], c["group"])
    if s["bias"] is not None:
        z = z + s["bias"]
    y = _act(z[:, :m], c["act"]) * z[:, m:] if c["gated"] else _act(z, c["act"])
    if s["R"] is not None:
        y = y + c["rho"] * _f(s["R"])
    return {"Y": y.to(t)}


# ---- the library's calls --------------------------------------------------------------------------------------------
def _code(g, act):
    return {"none": g.ACT_NONE, "relu": g.ACT_RELU, "gelu": g.ACT_GELU, "silu": g.ACT_SILU}[act]


def _own_gated(c, s):
    import paper_2005_03300_amd as g
    act = _code(g, c["act"])
    if c["pass_"] == "forward":
        g.gcn_gated_forward(s["X"], s["W"], s["H"], bias=s["bias"], act=act, Z=s["Z"])
        return {"H": s["H"], "Z": s["Z"]} if c["keep"] else {"H": s["H"]}
    g.gcn_gated_backward(s["X"], s["W"], s["Z"], s["dH"], s["dZ"], dX=s["dX"], dW=s["dW"], dbias=s["dbias"], act=act, H=s["H"])
    return {k: s[k] for k in ("H", "dX", "dW", "dbias") if s[k] is not None}


def _own_checkpoint(c, s):
    import paper_2005_03300_amd as g
    if c["pass_"] == "restore":
        g.gcn_checkpoint_pack(s["X"], *s["held"])
        g.gcn_checkpoint_unpack(*s["held"], s["back"])
        return {"X": s["back"], "scales": s["held"][1]}
    g.gcn_checkpoint_linear_backward(s["X"], s["W"], s["Z"], s["dY"], s["dZ"], dX=s["dX"], dW=s["dW"], dbias=s["dbias"],
                                     act=_code(g, c["act"]), dR=s["dR"], rho=c["rho"])
    return {k: s[k] for k in ("dX", "dW", "dbias", "dR") if s[k] is not None}


def _own_linear4(c, s):
    import paper_2005_03300_amd as g
    if c["pass_"] == "restore":
        g.gcn_linear4_pack(s["W"], *s["held"], group=c["group"])
        g.gcn_linear4_unpack(*s["held"], s["back"], group=c["group"])
        return {"W": s["back"], "scales": s["held"][1]}
    g.gcn_linear4_forward(s["X"], *s["held"], s["Y"], group=c["group"], bias=s["bias"], act=_code(g, c["act"]), R=s["R"], rho=c["rho"],
                          gated=c["gated"])
    return {"Y": s["Y"]}


_PLAIN = {"gated": _plain_gated, "checkpoint": _plain_checkpoint, "linear4": _plain_linear4}
_OWN = {"gated": _own_gated, "checkpoint": _own_checkpoint, "linear4": _own_linear4}


def run(state):
    c = state["case"]
    return (_OWN if own else _PLAIN)[c["op"]](c, state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def _held_bytes(n, f):
    return n * f + 2 * n * -(-f // _GROUP)


def work(case):
    c, e, n, k = case, _BYTES[case["type"]], case["n"], case["k"]
    if c["op"] == "gated":
        m = c["m"]
        if c["pass_"] == "forward":
            return {"bytes": e * (n * k + 2 * k * m + n * m * (3 if c["keep"] else 1)) + 8 * m * bool(c["bias"]), "flops": 4 * n * k * m}
        kept = _held_bytes(n, k) + _held_bytes(n, 2 * m) if c["held8"] else e * (n * k + 2 * n * m)
        return {"bytes": kept + e * (2 * n * m + n * k + 4 * k * m) + 8 * m * bool(c["bias"]), "flops": 8 * n * k * m}
    if c["op"] == "checkpoint":
        if c["pass_"] == "restore":
            return {"bytes": 2 * e * n * k + _held_bytes(n, k), "flops": 6 * n * k}
        m = c["m"]
        kept = _held_bytes(n, k) + (_held_bytes(n, m) if c["act"] != "none" else 0)
        return {"bytes": kept + e * (n * m * (1 + (c["rho"] != 1.0)) + n * k + 2 * k * m) + 4 * m * bool(c["bias"]), "flops": 4 * n * k * m}
    m, group = c["m"], c["group"]
    cols = 2 * m if c["gated"] else m
    held = cols * (4 * -(-k // 8) + 2 * -(-k // group))
    if c["pass_"] == "restore":
        return {"bytes": 2 * e * k * cols + held, "flops": 20 * k * cols}
    return {"bytes": held + e * (n * k + n * m * (1 + bool(c["residual"]))) + 4 * cols * bool(c["bias"]), "flops": 2 * n * k * cols}


# ---- from the definitions, in 64 bits -------------------------------------------------------------------------------
def _d(t):
    return None if t is None else t.double()


_CURVES = {"none": lambda z: z, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}


def _exact_scales(most, steps):
    m, e = torch.frexp(most / steps)                               # m in [1/2, 1): eight bits of it, rounded up
    power = ((e.long() + (1023 - 8)) << 52).view(torch.float64)    # 2^(e - 8), to the last bit
    return (torch.ceil(m * 256) * power).clamp(min=2.0 ** -126)


def _exact_matrix(held, t):
    """The matrix that a pass has in hand, in 64 bits."""
    if not isinstance(held, tuple):
        return _d(held)
    c, s = held
    at = torch.arange(c.shape[1], device=c.device) // _GROUP
    return (c.double() * s.double()[:, at]).to(t).double()


def _exact_gated(c, s):
    t, m, f = _TYPES[c["type"]], c["m"], _CURVES[c["act"]]
    W = _d(s["W"])
    if c["pass_"] == "forward":
        z = _d(s["X"]) @ W if s["bias"] is None else torch.addmm(s["bias"].double(), _d(s["X"]), W)
        h = f(z[:, :m]) * z[:, m:]
        return {"H": h, "Z": z} if c["keep"] else {"H": h}
    z = _exact_matrix(s["Z"], t).requires_grad_()
    g, u = z.split(m, 1)
    h = f(g) * u
    dZ, = torch.autograd.grad(h, z, _d(s["dH"]))
    out = {"H": h.detach(), "dX": dZ @ W.t(), "dW": _exact_matrix(s["X"], t).t() @ dZ}
    if s["dbias"] is not None:
        out["dbias"] = dZ.sum(0)
    return out


def _exact_checkpoint(c, s):
    t = _TYPES[c["type"]]
    if c["pass_"] == "restore":
        X = _d(s["X"])
        n, k = X.shape
        x = torch.nn.functional.pad(X, (0, -k % _GROUP)).view(n, -1, _GROUP)
        scale = _exact_scales(x.abs().max(2).values, 127)
        x = (x / scale[:, :, None]).round() * scale[:, :, None]
        return {"X": x.view(n, -1)[:, :k].to(t).double(), "scales": scale}
    z = _exact_matrix(s["Z"], t).requires_grad_()
    dZ, = torch.autograd.grad(_CURVES[c["act"]](z), z, _d(s["dY"]))
    out = {"dX": dZ @ _d(s["W"]).t(), "dW": _exact_matrix(s["X"], t).t() @ dZ, "dbias": dZ.sum(0), "dR": c["rho"] * _d(s["dY"])}
    return {k: v for k, v in out.items() if s[k] is not None}


def _exact_linear4(c, s):
    t, k, m, group = _TYPES[c["type"]], c["k"], c["m"], c["group"]
    levels = torch.tensor([x for x in _LEVELS] + [-x for x in _LEVELS], dtype=torch.float64, device="cuda")
    if c["pass_"] == "restore":
        W = _d(s["W"])
        w = torch.nn.functional.pad(W, (0, 0, 0, -k % group)).view(-1, group, W.shape[1])
        scale = _exact_scales(w.abs().max(1).values, 6)
        x = w / scale[:, None]
        # the nearest multiple of 1/2 below 2, of 1 up to 4 and of 2 beyond: of two that are as near, the even one
        a = x.abs()
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        x = torch.copysign((a / step).round() * step, x) * scale[:, None]
        return {"W": x.reshape(-1, W.shape[1])[:k].to(t).double(), "scales": scale}
    q, scale = s["held"]
    at = torch.arange(k, device="cuda")
    W = levels[((q[at // 8] >> (at % 8 * 4).int()[:, None]) & 15).long()] * scale.double()[at // group]
    z = _d(s["X"]) @ W
    if s["bias"] is not None:
        z = z + s["bias"].double()
    f = _CURVES[c["act"]]
    y = f(z[:, :m]) * z[:, m:] if c["gated"] else f(z)
    return {"Y": y if s["R"] is None else torch.add(y, s["R"].double(), alpha=c["rho"])}


def exact(case, seed):
    s = prepare(case, seed)
    return {"gated": _exact_gated, "checkpoint": _exact_checkpoint, "linear4": _exact_linear4}[case["op"]](case, s)
