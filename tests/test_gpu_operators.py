"""The operators of residual networks (linear layer with its epilogue, norms around a block, distillation) against plain
implementations in 64 bits, through the C ABI.

Tolerances are bounds, element by element: a sum of K terms in 32 bits is off by at most K 2^-24 times the sum of the terms' absolute
values in any order, a result rounded to its type by half a unit in the last place (`UNIT`), and elementary functions by a few
2^-24.  Each test multiplies what its own formula is made of."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 1e-37, "bf16": 1e-37, "f16": 2.0 ** -24}      # below the smallest normal number a type's roundings are absolute
EPS = 2.0 ** -24
ALL = list(TYPES)


def lib():
    import paper_2005_03300_amd as g
    g.lib()
    return g


class Strided:
    """A rows x cols operand inside a larger buffer: `pad` elements between rows, `skip` in front, everything outside the operand
    holds NaN (inputs) or a mark (outputs), which must still be there afterwards."""

    def __init__(self, rows, cols, type_, pad=0, skip=0, value=None, mark=float("nan")):
        self.rows, self.cols, self.ld, self.skip = rows, cols, cols + pad, skip
        self.buffer = torch.full((skip + rows * self.ld + 64,), mark, dtype=TYPES[type_], device="cuda")
        self.t = self.buffer[skip:skip + rows * self.ld].view(rows, self.ld)[:, :cols]
        if value is not None:
            self.t.copy_(value)
        self.before = self.buffer.clone()

    def outside_is_untouched(self):
        a, b = self.buffer.clone(), self.before.clone()
        for x in (a, b):
            x[self.skip:self.skip + self.rows * self.ld].view(self.rows, self.ld)[:, :self.cols] = 0
        return torch.equal(torch.nan_to_num(a, nan=-7.0), torch.nan_to_num(b, nan=-7.0))


def out(rows, cols, type_, pad=0, skip=0):
    return Strided(rows, cols, type_, pad, skip, mark=3.0)


def normal(gen, shape, type_, scale=1.0):
    return (torch.randn(shape, generator=gen, dtype=torch.float64) * scale).to(TYPES[type_])


def gen_of(*key):
    seed = 0
    for k in key:
        for ch in str(k):
            seed = (seed * 131 + ord(ch)) % (1 << 31)
    return torch.Generator().manual_seed(seed)


def check(got, ref, tol, what):
    got = got.detach().double().cpu()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    fine = torch.isfinite(ref)
    assert torch.equal(fine, torch.isfinite(got)), f"{what}: finite in other places"
    off = (got - ref).abs()[fine]
    bound = tol.expand_as(ref)[fine] if torch.is_tensor(tol) else torch.full_like(off, tol)
    if off.numel():
        worst = int((off / bound.clamp(min=1e-300)).argmax())
        assert bool((off <= bound).all()), f"{what}: off by {off[worst]:.3e}, allowed {bound[worst]:.3e} ({int((off > bound).sum())} of {off.numel()})"


# ---- linear ---------------------------------------------------------------------------------------------------------
def act64(z, act):
    return {"none": lambda v: v, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[act](z)


def slope64(z, act):
    if act == "none":
        return torch.ones_like(z)
    z = z.clone().requires_grad_()
    g, = torch.autograd.grad(act64(z, act).sum(), z)
    return g


def code(g, act):
    return {"none": g.ACT_NONE, "relu": g.ACT_RELU, "gelu": g.ACT_GELU, "silu": g.ACT_SILU}[act]


SLOPE_MOST = 1.13      # of the slopes of all activations: gelu's at z = 1.41

# n, f_in, f_out, padding between rows, elements in front: single elements, one row, sizes below, at and above tiles and their depth, long sums that
# are split, many rows with few columns, and the reverse
LINEAR = [
    (1, 1, 1, 0, 0), (1, 64, 64, 0, 0), (1, 1000, 300, 0, 0), (2, 4096, 40, 8, 0), (3, 5, 7, 0, 1), (16, 512, 1024, 0, 0), (17, 33, 65, 3, 0), (33, 160, 96, 0, 8),
    (64, 64, 64, 0, 0), (65, 128, 129, 0, 0), (130, 602, 41, 0, 0), (256, 64, 256, 0, 0), (257, 96, 304, 16, 0), (1000, 37, 8, 0, 0),
    (2049, 72, 1608, 0, 0), (2049, 71, 1601, 1, 1), (4099, 136, 4096, 0, 0), (20001, 48, 24, 0, 0), (9, 3000, 17, 0, 0),
]
ACTS = ["none", "relu", "gelu", "silu"]


@pytest.mark.parametrize("type_", ALL)
@pytest.mark.parametrize("at", range(len(LINEAR)))
def test_linear_forward(type_, at):
    g = lib()
    n, K, N, pad, skip = LINEAR[at]
    act = ACTS[(at + ALL.index(type_)) % 4]
    bias, residual, keep = at % 3 != 0, at % 2 == 0, at % 4 != 1
    rho = 1.0 if at % 4 < 2 else -0.75
    gen = gen_of("linear", type_, at)
    X = Strided(n, K, type_, pad, skip, normal(gen, (n, K), type_))
    W = Strided(K, N, type_, pad, skip, normal(gen, (K, N), type_, K ** -0.5))
    b = normal(gen, (N,), "f32").cuda() if bias else None
    R = Strided(n, N, type_, pad, skip, normal(gen, (n, N), type_)) if residual else None
    Y, Z = out(n, N, type_, pad, skip), out(n, N, type_, pad, skip) if keep else None
    g.gcn_linear_forward(X.t, W.t, Y.t, bias=b, act=code(g, act), R=R.t if residual else None, rho=rho, Z=Z.t if keep else None)
    x, w = X.t.double().cpu(), W.t.double().cpu()
    z = x @ w + (b.double().cpu() if bias else 0)
    size = x.abs() @ w.abs() + (b.double().cpu().abs() if bias else 0)
    off = (K + 2) * EPS * size
    r = rho * R.t.double().cpu() if residual else torch.zeros_like(z)
    y = act64(z, act) + r
    if keep:
        check(Z.t, z, off + UNIT[type_] * (z.abs() + off) + TINY[type_], "Z")
        assert Z.outside_is_untouched()
    inner = SLOPE_MOST * off + 8 * EPS * (z.abs() + 1e-30) + 2 * EPS * r.abs()
    check(Y.t, y, inner + UNIT[type_] * (y.abs() + inner) + TINY[type_], "Y")
    assert Y.outside_is_untouched()
    again = out(n, N, type_, pad, skip)
    g.gcn_linear_forward(X.t, W.t, again.t, bias=b, act=code(g, act), R=R.t if residual else None, rho=rho)
    assert torch.equal(again.t, Y.t), "the same call gives other bits"


@pytest.mark.parametrize("type_", ALL)
@pytest.mark.parametrize("at", range(len(LINEAR)))
def test_linear_backward(type_, at):
    g = lib()
    n, K, N, pad, skip = LINEAR[at]
    act = ACTS[(at + 1 + ALL.index(type_)) % 4]
    rho = 0.5
    gen = gen_of("back", type_, at)
    X = Strided(n, K, type_, pad, skip, normal(gen, (n, K), type_))
    W = Strided(K, N, type_, pad, skip, normal(gen, (K, N), type_, K ** -0.5))
    Z = Strided(n, N, type_, pad, skip, normal(gen, (n, N), type_))
    dY = Strided(n, N, type_, pad, skip, normal(gen, (n, N), type_))
    dZ, dX, dW, dR = out(n, N, type_, pad, skip), out(n, K, type_, pad, skip), out(K, N, type_, pad, skip), out(n, N, type_, pad, skip)
    db = torch.empty(N, device="cuda")
    g.gcn_linear_backward(X.t, W.t, Z.t, dY.t, dZ.t, dX=dX.t, dW=dW.t, dbias=db, act=code(g, act), dR=dR.t, rho=rho)
    x, w, z, dy = (t.t.double().cpu() for t in (X, W, Z, dY))
    dz = dy * slope64(z, act)
    u = UNIT[type_]
    # the slope in 32 bits: its terms are at most |z| + 2; then rounded to the type, where there is a slope to multiply by
    near = 8 * EPS * (z.abs() + 2) * dy.abs()
    dz_off = torch.zeros_like(dz) if act == "none" else near + u * (dz.abs() + near) + TINY[type_]
    size = dz.abs() + dz_off

    def product(p, q, pq_off, terms):
        ref = p @ q
        off = pq_off
        return ref, off + u * (ref.abs() + off) + TINY[type_]
    ref, tol = product(dz, w.t(), dz_off @ w.t().abs() + (N + 2) * EPS * (size @ w.t().abs()), N)
    check(dX.t, ref, tol, "dX")
    ref, tol = product(x.t(), dz, x.t().abs() @ dz_off + (n + 2) * EPS * (x.t().abs() @ size), n)
    check(dW.t, ref, tol, "dW")
    check(db, dz.sum(0), near.sum(0) * (act != "none") + (n + 2) * EPS * (dz.abs() + near).sum(0) + 1e-37, "dbias")
    check(dR.t, rho * dy, u * rho * dy.abs() + TINY[type_], "dR")
    for t in (dZ, dX, dW, dR):
        assert t.outside_is_untouched()
    # each gradient by itself is the same one
    for one in ("dX", "dW", "dbias", "dR"):
        alone = dict(dX=torch.empty_like(dX.t), dW=torch.empty_like(dW.t), dbias=torch.empty_like(db), dR=torch.empty_like(dR.t))[one]
        g.gcn_linear_backward(X.t, W.t, Z.t, dY.t, dZ.t, act=code(g, act), rho=rho, **{one: alone})
        assert torch.equal(alone, dict(dX=dX.t, dW=dW.t, dbias=db, dR=dR.t)[one]), one


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_linear_gradient_against_differences(act):
    """Along a random direction of all inputs, against the quotient of differences of the plain form in 64 bits (step 1e-5: the quotient is
    off by about 1e-9)."""
    g = lib()
    n, K, N, rho = 37, 50, 29, 0.5
    gen = gen_of("differences", act)
    X, W, R, C = (normal(gen, s, "f32") for s in ((n, K), (K, N), (n, N), (n, N)))
    W, b = W * K ** -0.5, normal(gen, (N,), "f32")
    D = [torch.randn(t.shape, generator=gen, dtype=torch.float64) for t in (X, W, b, R)]
    forms = [t.double() for t in (X, W, b, R)]

    def value(h):
        x, w, c, r = (t + h * d for t, d in zip(forms, D))
        return float((C.double() * (rho * r + act64(x @ w + c, act))).sum())
    quotient = (value(1e-5) - value(-1e-5)) / 2e-5
    dev = [t.cuda() for t in (X, W, b, R)]
    Y, Z, dZ = (torch.empty(n, N, device="cuda") for _ in range(3))
    g.gcn_linear_forward(dev[0], dev[1], Y, bias=dev[2], act=code(g, act), R=dev[3], rho=rho, Z=Z)
    grads = [torch.empty_like(t) for t in dev]
    g.gcn_linear_backward(dev[0], dev[1], Z, C.cuda(), dZ, dX=grads[0], dW=grads[1], dbias=grads[2], act=code(g, act), dR=grads[3], rho=rho)
    terms = [(gr.double().cpu() * d) for gr, d in zip(grads, D)]
    got, size = sum(float(t.sum()) for t in terms), sum(float(t.abs().sum()) for t in terms)
    assert abs(got - quotient) <= 100 * EPS * size + 1e-7 * abs(quotient) + 1e-7


@pytest.mark.parametrize("type_", ALL)
@pytest.mark.parametrize("n,K,N", [(5, 64, 48), (300, 200, 130), (4, 2048, 64)])
def test_linear_in_place_and_special_values(type_, n, K, N):
    """The residual's place takes the result; infinities and NaN stay in their rows and columns."""
    g = lib()
    gen = gen_of("special", type_, n)
    X, W = normal(gen, (n, K), type_).cuda(), normal(gen, (K, N), type_, K ** -0.5).cuda()
    R = normal(gen, (n, N), type_).cuda()
    Y = torch.empty_like(R)
    g.gcn_linear_forward(X, W, Y, act=g.ACT_SILU, R=R, rho=0.5)
    g.gcn_linear_forward(X, W, R, act=g.ACT_SILU, R=R, rho=0.5)
    assert torch.equal(R, Y)
    base = torch.empty_like(R)
    g.gcn_linear_forward(X, W, base)
    X[1, 3], X[2, K - 1] = float("nan"), float("inf")
    Y = torch.empty_like(R)
    g.gcn_linear_forward(X, W, Y)
    keep = [i for i in range(n) if i not in (1, 2)]
    assert torch.equal(Y[keep], base[keep])
    assert bool(torch.isnan(Y[1]).all())
    sign = torch.where(W[K - 1] > 0, 1, -1)
    there = W[K - 1] != 0
    assert torch.equal(Y[2][there].float(), (sign[there] * float("inf")).float())
    # ReLU keeps NaN, and so does its derivative
    g.gcn_linear_forward(X, W, Y, act=g.ACT_RELU)
    assert bool(torch.isnan(Y[1]).all()) and bool((Y[keep] >= 0).all())


@pytest.mark.parametrize("n,K,N", [(300, 200, 130), (2049, 72, 1608)])
def test_linear_fp32_keeps_its_bits_and_infinities(n, K, N):
    """Products of fp32 numbers keep 24 bits over the whole range of magnitudes; infinities, NaN and numbers next to the largest one in either operand give what
    fp32 products give, and change no other result."""
    g = lib()
    gen = gen_of("thirds", n)
    scale = torch.exp2(torch.randint(-20, 21, (n, K), generator=gen).double())
    X = (torch.randn(n, K, generator=gen, dtype=torch.float64) * scale).float().cuda()
    W = (torch.randn(K, N, generator=gen, dtype=torch.float64) * torch.exp2(torch.randint(-20, 21, (K, N), generator=gen).double())).float().cuda()
    Y = torch.empty(n, N, device="cuda")
    g.gcn_linear_forward(X, W, Y)
    x, w = X.double().cpu(), W.double().cpu()
    check(Y, x @ w, (K + 2) * EPS * (x.abs() @ w.abs()), "Y")
    x1, w1 = X.clone(), W.clone()
    big = torch.finfo(torch.float32).max
    x1[3, 1], x1[70, K - 1], x1[n - 1, 5], x1[140, 2] = float("inf"), float("-inf"), float("nan"), big
    w1[:, 4] *= 2.0 ** -40                                     # (so that the largest number's products are finite in one column)
    w1[6, N - 1] = float("inf")
    got = torch.empty_like(Y)
    g.gcn_linear_forward(x1, w1, got)
    rows, cols = [i for i in range(n) if i not in (3, 70, n - 1, 140)], [j for j in range(N) if j not in (4, N - 1)]
    assert torch.equal(got[rows][:, cols], Y[rows][:, cols])
    ref = x1.double().cpu() @ w1.double().cpu()
    ref = torch.where(ref.abs() > big, ref.sign() * float("inf"), ref)
    for i in (3, 70, n - 1):
        assert torch.equal(got[i].double().cpu().nan_to_num(7.0, 8.0, 9.0), ref[i].nan_to_num(7.0, 8.0, 9.0)), i
    assert torch.equal(torch.isfinite(got[140]).cpu(), torch.isfinite(ref[140])) and bool(torch.isfinite(got[140, 4]))
    size = x1.abs().double().cpu() @ w1.abs().double().cpu()
    assert abs(float(got[140, 4]) - float(ref[140, 4])) <= (K + 2) * EPS * float(size[140, 4])
    assert torch.equal(got[rows][:, N - 1].cpu().double().sign(), x1[rows][:, 6].cpu().double().sign()) and bool(torch.isinf(got[rows][:, N - 1]).all())
    # the gradients' products too
    dX, dW = torch.empty_like(X), torch.empty_like(W)
    dY = normal(gen, (n, N), "f32").cuda()
    g.gcn_linear_backward(X, W, None, dY, dX=dX, dW=dW)
    d1 = dY.clone()
    d1[5, 7] = float("inf")
    dX1, dW1 = torch.empty_like(X), torch.empty_like(W)
    g.gcn_linear_backward(X, W, None, d1, dX=dX1, dW=dW1)
    others = [i for i in range(n) if i != 5]
    assert torch.equal(dX1[others], dX[others]) and torch.equal(dX1[5].sign(), W[:, 7].sign()) and bool(torch.isinf(dX1[5]).all())
    others = [j for j in range(N) if j != 7]
    assert torch.equal(dW1[:, others], dW[:, others]) and torch.equal(dW1[:, 7].sign(), X[5].sign()) and bool(torch.isinf(dW1[:, 7]).all())


def test_linear_backward_in_place_of_its_inputs():
    g = lib()
    gen = gen_of("aliases")
    n, K, N = 70, 40, 56
    X, W = normal(gen, (n, K), "bf16").cuda(), normal(gen, (K, N), "bf16").cuda()
    Z, dY = normal(gen, (n, N), "bf16").cuda(), normal(gen, (n, N), "bf16").cuda()
    dZ, dX, dW = torch.empty_like(Z), torch.empty_like(X), torch.empty_like(W)
    g.gcn_linear_backward(X, W, Z, dY, dZ, dX=dX, dW=dW, act=g.ACT_GELU)
    for place in ("Z", "dY"):
        z, dy = Z.clone(), dY.clone()
        dx, dw = torch.empty_like(X), torch.empty_like(W)
        g.gcn_linear_backward(X, W, z, dy, z if place == "Z" else dy, dX=dx, dW=dw, act=g.ACT_GELU)
        assert torch.equal(dx, dX) and torch.equal(dw, dW)
    z, dy = Z.clone(), dY.clone()
    dx, dw = torch.empty_like(X), torch.empty_like(W)
    g.gcn_linear_backward(X, W, z, dy, z, dX=dx, dW=dw, act=g.ACT_GELU, dR=dy, rho=0.25)
    assert torch.equal(dx, dX) and torch.equal(dw, dW) and torch.equal(dy, (dY.float() * 0.25).bfloat16())


def test_linear_refusals():
    g = lib()
    X, W, Y = (torch.zeros(8, 8, device="cuda") for _ in range(3))

    def refused(f, text):
        with pytest.raises(g.GcnError) as e:
            f()
        assert e.value.code == -1 and text in str(e.value), str(e.value)
    L, now = g.lib(), g.binding._now
    fwd = lambda n=8, fi=8, fo=8, type_=0, act=0, x=X, w=W, y=Y, z=None, r=None, ldx=8: g.binding._check(L.gcn_linear_forward(
        n, fi, fo, type_, g.binding._at(x), ldx, g.binding._at(w), 8, None, act, g.binding._at(r), 8, 1.0, g.binding._at(z), 8, g.binding._at(y), 8, now()))
    refused(lambda: fwd(x=None), "NULL")
    refused(lambda: fwd(n=0), "positive")
    refused(lambda: fwd(fi=-1), "positive")
    with pytest.raises(g.GcnError) as e:
        fwd(fo=(1 << 30) + 1)
    assert e.value.code == -2
    refused(lambda: fwd(type_=3), "element type")
    refused(lambda: fwd(act=4), "activation")
    refused(lambda: fwd(ldx=7), "leading dimension")
    refused(lambda: fwd(y=X), "overlaps")
    refused(lambda: fwd(y=W), "overlaps")
    refused(lambda: fwd(z=Y), "overlaps")
    refused(lambda: fwd(r=Y.view(-1)[1:]), "overlaps")
    G, Z = torch.zeros(8, 8, device="cuda"), torch.zeros(8, 8, device="cuda")
    refused(lambda: g.gcn_linear_backward(X, W, None, G, None, dX=Y, act=g.ACT_GELU), "needs Z")
    refused(lambda: g.gcn_linear_backward(X, W, Z, G, None, dX=Y, act=g.ACT_GELU), "workspace")
    refused(lambda: g.gcn_linear_backward(None, W, Z, G, None, dW=Y), "NULL")
    refused(lambda: g.gcn_linear_backward(X, W, Z, G, None, dX=G), "overlaps")
    refused(lambda: g.gcn_linear_backward(X, W, None, G, None, dX=Y, dR=G), "overlaps")
    with pytest.raises(AssertionError):
        g.gcn_linear_forward(X, W.bfloat16(), Y)
    with pytest.raises(AssertionError):
        g.gcn_linear_forward(X.double(), W.double(), Y.double())


# ---- norms around a block -------------------------------------------------------------------------------------------
DEPTH = 160     # additions that one number goes through in a sum over a row: a lane's own, then in pairs, then the wavefronts'
NORM_EPS = 1e-5


def norm64(x, w, b, layer):
    mean = x.mean(1, keepdim=True) if layer else torch.zeros_like(x[:, :1])
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + NORM_EPS)
    hat = (x - mean) * rstd
    y = hat * w + (b if b is not None else 0)
    # how far a norm in 32 bits may be off: the mean by its additions, the deviation's relative error half of the variance's, the products
    size = (x.abs() + x.abs().mean(1, keepdim=True)) * rstd
    off = w.abs() * (DEPTH * EPS * x.abs().mean(1, keepdim=True) * rstd + 4 * EPS * size + hat.abs() * DEPTH * EPS) + 2 * EPS * y.abs()
    return y, mean, rstd, off


# rows, width, padding, elements in front: one element, widths around 16 bytes, a wavefront's rows, a workgroup's, and longer than registers hold
NORM = [(1, 1, 0, 0), (1, 4096, 0, 0), (3, 5, 0, 1), (70, 16, 0, 0), (129, 33, 1, 0), (33, 128, 0, 0), (18, 301, 0, 0), (5, 511, 1, 3), (7, 1024, 8, 0),
        (4, 2050, 0, 0), (3, 4097, 0, 0), (3, 8192, 0, 0), (2, 9001, 0, 1), (2, 16384, 0, 0), (2, 20003, 0, 0)]


def norm_operands(type_, at, key):
    n, f, pad, skip = NORM[at]
    gen = gen_of(key, type_, at)
    layer, gate, post = at % 2 == 0, [f, 1, 0][at % 3], at % 5 != 3
    o = dict(n=n, f=f, layer=layer, gate=gate, post=post)
    make = lambda scale=1.0: Strided(n, f, type_, pad, skip, normal(gen, (n, f), type_, scale))
    o["X"], o["U"] = make(), make(2.0)
    o["A"] = Strided(n, gate, type_, pad, skip, normal(gen, (n, gate), type_)) if gate else None
    vec = lambda c=1.0: (c + 0.2 * torch.randn(f, generator=gen, dtype=torch.float64)).float()
    o["scale"] = vec(0.3) if at % 4 != 2 else None
    o["w_post"] = vec() if post else None
    o["b_post"] = vec(0.0) if post and layer else None
    o["w_pre"] = vec()
    o["b_pre"] = vec(0.0) if layer else None
    return o, gen, pad, skip


def cuda(t):
    return None if t is None else t.cuda()


def d64(t):
    return None if t is None else (t.t if isinstance(t, Strided) else t).double().cpu()


def block64(o, X=None):
    """The plain forward pass, and how far one in 32 bits may be off X' and H."""
    U, A = d64(o["U"]), d64(o["A"])
    gate = torch.sigmoid(A) if A is not None else torch.ones_like(U)
    scale = d64(o["scale"]) if o["scale"] is not None else torch.ones(o["f"], dtype=torch.float64)
    v, um, ur, v_off = (U, None, None, torch.zeros_like(U))
    if o["post"]:
        v, um, ur, v_off = norm64(U, d64(o["w_post"]), d64(o["b_post"]), o["layer"])
    step = scale * gate * v
    x = d64(o["X"]) + step
    x_off = (scale * gate).abs() * v_off + 12 * EPS * step.abs() + EPS * x.abs()
    h, xm, xr, h_off = norm64(x, d64(o["w_pre"]), d64(o["b_pre"]), o["layer"])
    # the norm of a row that is off: three times as far, relative to its deviation, covers the row's own mean and deviation
    h_off = h_off + d64(o["w_pre"]).abs() * xr * (x_off + (1 + ((x - xm) * xr).abs()) * x_off.max(1, keepdim=True).values) * 2
    return x, x_off, h, h_off, um, ur, xm, xr


@pytest.mark.parametrize("type_", ALL)
@pytest.mark.parametrize("at", range(len(NORM)))
def test_block_norm_forward(type_, at):
    g = lib()
    o, gen, pad, skip = norm_operands(type_, at, "norm")
    n, f = o["n"], o["f"]
    kind = g.NORM_LAYER if o["layer"] else g.NORM_RMS
    Xo, H, stats = out(n, f, type_, pad, skip), out(n, f, type_, pad, skip), torch.full((n, 4), 9.0, device="cuda")
    args = dict(w_pre=cuda(o["w_pre"]), b_pre=cuda(o["b_pre"]), A=o["A"].t if o["gate"] else None, scale=cuda(o["scale"]),
                w_post=cuda(o["w_post"]), b_post=cuda(o["b_post"]), kind=kind, eps=NORM_EPS)
    g.gcn_block_norm_forward(o["X"].t, o["U"].t, Xo.t, H.t, stats=stats, **args)
    x, x_off, h, h_off, um, ur, xm, xr = block64(o)
    u = UNIT[type_]
    check(Xo.t, x, x_off + u * (x.abs() + x_off) + TINY[type_], "X'")
    check(H.t, h, h_off + u * (h.abs() + h_off) + TINY[type_], "H")
    assert Xo.outside_is_untouched() and H.outside_is_untouched()
    U = d64(o["U"])
    if o["post"]:
        check(stats[:, 0:1], um, DEPTH * EPS * U.abs().mean(1, keepdim=True) + 1e-37, "mean of U")
        check(stats[:, 1:2], ur, DEPTH * EPS * ur, "deviation of U")
    else:
        assert bool((stats[:, :2] == 0).all())
    far = x_off.max(1, keepdim=True).values
    check(stats[:, 2:3], xm, DEPTH * EPS * x.abs().mean(1, keepdim=True) + far + 1e-37, "mean of X'")
    check(stats[:, 3:4], xr, DEPTH * EPS * xr + 2 * xr * xr * far, "deviation of X'")
    # in place of the inputs, and the two results one at a time
    X2, U2 = o["X"].t.clone(), o["U"].t.clone()
    g.gcn_block_norm_forward(X2, U2, X2, U2, **args)
    assert torch.equal(X2, Xo.t) and torch.equal(U2, H.t)
    only = torch.empty_like(X2)
    g.gcn_block_norm_forward(o["X"].t, o["U"].t, None, only, **args)
    assert torch.equal(only, H.t)
    behind = {k: v for k, v in args.items() if k not in ("w_pre", "b_pre")}
    g.gcn_block_norm_forward(o["X"].t, o["U"].t, only, None, **behind)
    assert torch.equal(only, Xo.t)
    # in front of a first block
    g.gcn_block_norm_forward(o["X"].t, H=only, w_pre=args["w_pre"], b_pre=args["b_pre"], kind=kind, eps=NORM_EPS)
    ref, _, _, off = norm64(d64(o["X"]), d64(o["w_pre"]), d64(o["b_pre"]), o["layer"])
    check(only, ref, off + u * (ref.abs() + off) + TINY[type_], "norm alone")


def unit_gradient64(gw, hat, rstd, layer):
    along = (gw * hat).mean(1, keepdim=True)
    mean = gw.mean(1, keepdim=True) if layer else torch.zeros_like(along)
    size = rstd * (gw.abs() + hat.abs() * (gw * hat).abs().mean(1, keepdim=True) + gw.abs().mean(1, keepdim=True))
    return rstd * (gw - hat * along - mean), size


@pytest.mark.parametrize("type_", ALL)
@pytest.mark.parametrize("at", range(len(NORM)))
def test_block_norm_backward(type_, at):
    g = lib()
    o, gen, pad, skip = norm_operands(type_, at, "normback")
    n, f, layer = o["n"], o["f"], o["layer"]
    kind = g.NORM_LAYER if layer else g.NORM_RMS
    Xo = Strided(n, f, type_, pad, skip, normal(gen, (n, f), type_, 1.3))
    dXo, dH = (Strided(n, f, type_, pad, skip, normal(gen, (n, f), type_)) for _ in range(2))
    xo, U, dxo, dh = d64(Xo), d64(o["U"]), d64(dXo), d64(dH)
    stats64 = torch.zeros(n, 4, dtype=torch.float64)
    if o["post"]:
        _, stats64[:, 0:1], stats64[:, 1:2], _ = norm64(U, d64(o["w_pre"]), None, layer)
    _, stats64[:, 2:3], stats64[:, 3:4], _ = norm64(xo, d64(o["w_pre"]), None, layer)
    stats = stats64.float().cuda()
    um, ur, xm, xr = stats.double().cpu().split(1, dim=1)     # what the call is given
    dX, dU = out(n, f, type_, pad, skip), out(n, f, type_, pad, skip)
    dA = out(n, o["gate"], type_, pad, skip) if o["gate"] else None
    vec = lambda there: torch.full((f,), 7.0, device="cuda") if there else None
    v = dict(dscale=vec(o["scale"] is not None), dw_post=vec(o["post"]), db_post=vec(o["b_post"] is not None), dw_pre=vec(True), db_pre=vec(layer))
    common = dict(w_pre=cuda(o["w_pre"]), A=o["A"].t if o["gate"] else None, scale=cuda(o["scale"]), w_post=cuda(o["w_post"]),
                  b_post=cuda(o["b_post"]), kind=kind)
    g.gcn_block_norm_backward(o["U"].t, Xo.t, stats, dXo.t, dH.t, dX.t, dU.t, dA=dA.t if dA else None, **v, **common)
    u = UNIT[type_]
    K = 4 * DEPTH * EPS          # every gradient goes through at most two sums over the row and some products: relative to absolute values
    w_pre = d64(o["w_pre"])
    xhat = (xo - xm) * xr
    xsize = (xo.abs() + xm.abs()) * xr
    step, size = unit_gradient64(dh * w_pre, xhat, xr, layer)
    dx = dxo + step
    size = dxo.abs() + unit_gradient64((dh * w_pre).abs(), xsize, xr, True)[1]
    check(dX.t, dx, K * size + u * dx.abs() + TINY[type_], "dX")
    scale = d64(o["scale"]) if o["scale"] is not None else torch.ones(f, dtype=torch.float64)
    A = d64(o["A"])
    gate = torch.sigmoid(A) if A is not None else torch.ones(n, 1, dtype=torch.float64)
    w = d64(o["w_post"]) if o["post"] else torch.ones(f, dtype=torch.float64)
    b = d64(o["b_post"]) if o["b_post"] is not None else torch.zeros(f, dtype=torch.float64)
    uhat = (U - um) * ur if o["post"] else U
    usize = (U.abs() + um.abs()) * ur if o["post"] else U.abs()
    val, vsize = uhat * w + b, usize * w.abs() + b.abs()
    if A is not None:
        da, dasize = dx * scale * val * gate * (1 - gate), size * scale.abs() * vsize * gate
        if o["gate"] != f:
            da, dasize = da.sum(1, keepdim=True), dasize.sum(1, keepdim=True)
        check(dA.t, da, K * dasize + u * da.abs() + TINY[type_], "dA")
    dv, dvsize = dx * scale * gate, size * scale.abs() * gate
    du, dusize = dv * w, dvsize * w.abs()
    if o["post"]:
        du = unit_gradient64(dv * w, uhat, ur, layer)[0]
        dusize = unit_gradient64(dvsize * w.abs(), usize, ur, True)[1]
    check(dU.t, du, K * dusize + u * du.abs() + TINY[type_], "dU")
    KV = K + (n + 2) * EPS
    sums = dict(dscale=(dx * gate * val, size * gate * vsize), dw_post=(dv * uhat, dvsize * usize), db_post=(dv, dvsize),
                dw_pre=(dh * xhat, dh.abs() * xsize), db_pre=(dh, dh.abs()))
    for name, (terms, sizes) in sums.items():
        if v[name] is not None:
            check(v[name], terms.sum(0), KV * sizes.sum(0) + 1e-37, name)
    for t in (dX, dU, dA):
        assert t is None or t.outside_is_untouched()
    # in place of the inputs; the vectors' gradients are the same bits with or without the matrices'
    c = dict(common, A=o["A"].t.clone() if o["gate"] else None)
    U2, dxo2 = o["U"].t.clone(), dXo.t.clone()
    g.gcn_block_norm_backward(U2, Xo.t, stats, dxo2, dH.t, U2, dxo2, dA=c["A"], **c)
    assert torch.equal(U2, dX.t) and torch.equal(dxo2, dU.t) and (dA is None or torch.equal(c["A"], dA.t))
    v2 = {k: None if t is None else torch.empty_like(t) for k, t in v.items()}
    g.gcn_block_norm_backward(o["U"].t, Xo.t, stats, dXo.t, dH.t, **v2, **common)
    assert all(t is None or torch.equal(t, v[k]) for k, t in v2.items())


@pytest.mark.parametrize("f", [6, 300, 4100, 9000])
@pytest.mark.parametrize("layer", [False, True])
def test_block_norm_biases_go_with_either_norm(f, layer):
    """Biases with the root-mean-square norm, and a layer norm without any; forward, and backward by differentiation of the plain form."""
    g = lib()
    gen = gen_of("biases", f, layer)
    n, kind = 7, g.NORM_LAYER if layer else g.NORM_RMS
    X, U, A, C, E = (normal(gen, (n, f), "f32") for _ in range(5))
    w, wp = (1 + 0.2 * torch.randn(f, generator=gen) for _ in range(2))
    b, bp = (None, None) if layer else (0.3 * torch.randn(f, generator=gen) for _ in range(2))
    leaf = {k: t.double().requires_grad_() for k, t in dict(X=X, U=U, A=A, w=w, wp=wp, b=b, bp=bp).items() if t is not None}

    def unit(x):
        x = x - x.mean(1, keepdim=True) if layer else x
        return x / torch.sqrt((x * x).mean(1, keepdim=True) + NORM_EPS)
    x = leaf["X"] + torch.sigmoid(leaf["A"]) * (unit(leaf["U"]) * leaf["wp"] + leaf.get("bp", 0))
    h = unit(x) * leaf["w"] + leaf.get("b", 0)
    want = dict(zip(leaf, torch.autograd.grad((C.double() * x).sum() + (E.double() * h).sum(), list(leaf.values()))))
    dev = {k: t.cuda() for k, t in dict(X=X, U=U, A=A, w=w, wp=wp, b=b, bp=bp).items() if t is not None}
    Xo, H, stats = torch.empty(n, f, device="cuda"), torch.empty(n, f, device="cuda"), torch.empty(n, 4, device="cuda")
    g.gcn_block_norm_forward(dev["X"], dev["U"], Xo, H, w_pre=dev["w"], b_pre=dev.get("b"), A=dev["A"], w_post=dev["wp"], b_post=dev.get("bp"),
                             stats=stats, kind=kind, eps=NORM_EPS)
    size = 4 * DEPTH * EPS * (1 + f ** 0.5)                   # of numbers of about 1, in rows whose largest are some times that
    check(Xo, x.detach(), torch.full((1, 1), size, dtype=torch.float64), "X'")
    check(H, h.detach(), torch.full((1, 1), size, dtype=torch.float64), "H")
    got = {k: torch.empty_like(t) for k, t in dev.items()}
    g.gcn_block_norm_backward(dev["U"], Xo, stats, C.cuda(), E.cuda(), got["X"], got["U"], w_pre=dev["w"], A=dev["A"], dA=got["A"],
                              w_post=dev["wp"], b_post=dev.get("bp"), dw_post=got["wp"], db_post=got.get("bp"), dw_pre=got["w"],
                              db_pre=got.get("b"), kind=kind)
    for k, t in want.items():
        check(got[k], t, torch.full((1,) * t.dim(), 4 * size, dtype=torch.float64), "d" + k)


@pytest.mark.parametrize("f", [48, 5000])
def test_block_norm_gradients_of_one_side(f):
    """Only dX', only dH, and no block."""
    g = lib()
    gen = gen_of("sides", f)
    n = 9
    X, U, A, C = (normal(gen, (n, f), "f32").cuda() for _ in range(4))
    w, wp = (1 + 0.1 * torch.randn(f, generator=gen)).cuda(), (1 + 0.1 * torch.randn(f, generator=gen)).cuda()
    Xo, H, stats = torch.empty_like(X), torch.empty_like(X), torch.empty(n, 4, device="cuda")
    g.gcn_block_norm_forward(X, U, Xo, H, w_pre=w, A=A, w_post=wp, stats=stats, kind=g.NORM_LAYER)
    zero = torch.zeros_like(C)
    for d in (dict(dXout=C, dH=None), dict(dXout=None, dH=C)):
        got, want = [[torch.empty_like(X) for _ in range(3)] for _ in range(2)]
        g.gcn_block_norm_backward(U, Xo, stats, d["dXout"], d["dH"], got[0], got[1], w_pre=w if d["dH"] is not None else None, A=A, dA=got[2],
                                  w_post=wp, kind=g.NORM_LAYER)
        full = {k: zero if t is None else t for k, t in d.items()}
        g.gcn_block_norm_backward(U, Xo, stats, full["dXout"], full["dH"], want[0], want[1], w_pre=w, A=A, dA=want[2], w_post=wp,
                                  kind=g.NORM_LAYER)
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    alone, dw = torch.empty_like(X), torch.empty(f, device="cuda")
    g.gcn_block_norm_backward(None, Xo, stats, None, C, alone, w_pre=w, dw_pre=dw, kind=g.NORM_LAYER)
    assert torch.equal(alone, want[0])


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("gate", [1, 0])
def test_block_norm_gradient_against_differences(layer, gate):
    """As for the linear layer: the plain form's quotient in 64 bits along a random direction of every input."""
    g = lib()
    n, f = 11, 77
    gen = gen_of("normdiff", layer, gate)
    mats = dict(X=normal(gen, (n, f), "f32"), U=normal(gen, (n, f), "f32", 2.0), A=normal(gen, (n, 1 if gate else f), "f32"))
    vecs = {k: 1 + 0.2 * torch.randn(f, generator=gen) for k in ("scale", "w_post", "w_pre")}
    if layer:
        vecs.update({k: 0.2 * torch.randn(f, generator=gen) for k in ("b_post", "b_pre")})
    every = {**mats, **vecs}
    D = {k: torch.randn(t.shape, generator=gen, dtype=torch.float64) for k, t in every.items()}
    C, E = (torch.randn(n, f, generator=gen) for _ in range(2))

    def value(h):
        o = {k: t.double() + h * D[k] for k, t in every.items()}
        v = norm64(o["U"], o["w_post"], o.get("b_post"), layer)[0]
        x = o["X"] + o["scale"] * torch.sigmoid(o["A"]) * v
        return float((C.double() * x).sum() + (E.double() * norm64(x, o["w_pre"], o.get("b_pre"), layer)[0]).sum())
    quotient = (value(1e-5) - value(-1e-5)) / 2e-5
    dev = {k: t.cuda() for k, t in every.items()}
    kind = g.NORM_LAYER if layer else g.NORM_RMS
    Xo, H, stats = torch.empty(n, f, device="cuda"), torch.empty(n, f, device="cuda"), torch.empty(n, 4, device="cuda")
    g.gcn_block_norm_forward(dev["X"], dev["U"], Xo, H, stats=stats, kind=kind, eps=NORM_EPS, **{k: dev[k] for k in every if k not in ("X", "U")})
    grad = {k: torch.empty_like(t) for k, t in dev.items()}
    g.gcn_block_norm_backward(dev["U"], Xo, stats, C.cuda(), E.cuda(), grad["X"], grad["U"], dA=grad["A"], kind=kind,
                              **{k: dev[k] for k in every if k in ("A", "scale", "w_post", "b_post", "w_pre")},
                              **{"d" + k: grad[k] for k in vecs})
    terms = [grad[k].double().cpu() * D[k] for k in every]
    got, size = sum(float(t.sum()) for t in terms), sum(float(t.abs().sum()) for t in terms)
    assert abs(got - quotient) <= 4 * DEPTH * EPS * size + 1e-6 * abs(quotient)


def test_block_norm_special_rows():
    """A row of zeros (its deviation is that of eps alone), one of a single large value, NaN and infinity in their rows only."""
    g = lib()
    n, f = 6, 100
    gen = gen_of("rows")
    X, U = normal(gen, (n, f), "f32"), normal(gen, (n, f), "f32")
    X[0], U[0] = 0, 0
    U[1] = 1e18
    X, U, w = X.cuda(), U.cuda(), torch.ones(f, device="cuda")
    Xo, H = torch.empty_like(X), torch.empty_like(X)
    g.gcn_block_norm_forward(X, U, Xo, H, w_pre=w, w_post=w, kind=g.NORM_LAYER)
    assert bool((Xo[0] == 0).all()) and bool((H[0] == 0).all()) and bool(torch.isfinite(H[2:]).all())
    g.gcn_block_norm_forward(X, U, Xo, H, w_pre=w, w_post=w)
    assert bool(torch.isfinite(H).all()) and float((Xo[1] - X[1] - 1).abs().max()) < 1e-5
    base = H.clone()
    U[3, 7], X[4, 1] = float("nan"), float("inf")
    g.gcn_block_norm_forward(X, U, Xo, H, w_pre=w, w_post=w)
    assert torch.equal(H[[0, 1, 2, 5]], base[[0, 1, 2, 5]]) and bool(torch.isnan(H[3]).all())
    assert not bool(torch.isfinite(H[4, 1]))


def test_block_norm_refusals():
    g = lib()
    t = lambda *s: torch.zeros(*s, device="cuda")
    X, U, Xo, H, w, stats = t(4, 8), t(4, 8), t(4, 8), t(4, 8), t(8), t(4, 4)

    def refused(f, text):
        with pytest.raises(g.GcnError) as e:
            f()
        assert e.value.code == -1 and text in str(e.value), str(e.value)
    refused(lambda: g.gcn_block_norm_forward(X, U, None, None), "NULL")
    refused(lambda: g.gcn_block_norm_forward(X, U, Xo, H), "go together")
    refused(lambda: g.gcn_block_norm_forward(X, None, None, H, w_pre=w, scale=w), "need U")
    refused(lambda: g.gcn_block_norm_forward(X, U, Xo, H, w_pre=w, b_post=w), "without w_post")
    refused(lambda: g.gcn_block_norm_forward(X, U, Xo, H, w_pre=w, kind=2), "unknown norm")
    refused(lambda: g.gcn_block_norm_forward(X, U, Xo, H, w_pre=w, eps=-1.0), "eps")
    refused(lambda: g.gcn_block_norm_forward(X, U, Xo, H, w_pre=w, A=t(4, 3)), "1 or f")
    refused(lambda: g.gcn_block_norm_forward(X, U, Xo, Xo, w_pre=w), "overlaps")
    refused(lambda: g.gcn_block_norm_forward(X, U, Xo, H, w_pre=w, stats=X.view(8, 4)[:4]), "overlaps")
    refused(lambda: g.gcn_block_norm_backward(U, Xo, stats, X, None, H, w_pre=w, dw_pre=t(8)), "need dH")
    refused(lambda: g.gcn_block_norm_backward(U, None, stats, None, X, H, w_pre=w), "X'")
    refused(lambda: g.gcn_block_norm_backward(U, Xo, stats, X, None, H, dw_post=t(8)), "not there")
    refused(lambda: g.gcn_block_norm_backward(None, Xo, stats, X, None, H, Xo), "need U")
    refused(lambda: g.gcn_block_norm_backward(U, Xo, stats, X, X, H, H, w_pre=w), "overlaps")
    L = g.lib()
    rc = L.gcn_block_norm_forward(0, 8, 0, 0, 1e-5, X.data_ptr(), 8, None, 0, None, 0, 0, None, None, None, w.data_ptr(), None, None, 0, H.data_ptr(), 8, None, 0)
    assert rc == -1
    rc = L.gcn_block_norm_forward(4, 8, 5, 0, 1e-5, X.data_ptr(), 8, None, 0, None, 0, 0, None, None, None, w.data_ptr(), None, None, 0, H.data_ptr(), 8, None, 0)
    assert rc == -1
    rc = L.gcn_block_norm_forward(4, 8, 0, 0, 1e-5, X.data_ptr(), 7, None, 0, None, 0, 0, None, None, None, w.data_ptr(), None, None, 0, H.data_ptr(), 8, None, 0)
    assert rc == -1


# ---- distillation ---------------------------------------------------------------------------------------------------
# rows, classes, list, padding, elements in front
DISTILL = [(1, 1, 1, 0, 0), (1, 2, 2, 0, 0), (300, 8, 3, 0, 0), (67, 16, 16, 1, 0), (129, 17, 4, 0, 1), (1000, 41, 8, 0, 0), (70, 64, 5, 0, 0), (19, 128, 64, 8, 0),
           (9, 129, 70, 0, 0), (7, 513, 64, 1, 1), (5, 2049, 200, 0, 0), (3, 5000, 64, 0, 0), (3, 9000, 33, 0, 0), (2, 33001, 1500, 0, 0), (2, 66000, 64, 0, 0),
           (2, 140001, 64, 0, 0)]


def distill64(Z, top, t, y, T, wt, wl, m, scale):
    """Loss and gradient row by row from the definitions, and the sizes of what they are made of."""
    n, C = Z.shape
    lq = torch.log_softmax(Z / T, 1)
    q, soft = lq.exp(), torch.softmax(Z, 1)
    ls = torch.log_softmax(Z, 1)
    loss, size = 0.0, 0.0
    G = torch.zeros_like(Z)
    Gsize = torch.zeros_like(Z)
    for i in range(n):
        use = (top[i] >= 0) & (top[i] < C) & (t[i] != -math.inf)
        if bool(use.any()):
            at, lp = top[i][use], torch.log_softmax(t[i][use] / T, 0)
            p = lp.exp()
            terms = torch.where(p > 0, p * (lp - lq[i][at]), torch.zeros_like(p))
            loss += wt * T * T * float(terms.sum())
            size += wt * T * T * float((p * (lp.abs() + torch.where(p > 0, lq[i][at].abs(), torch.zeros_like(p)) + t[i][use].abs() / T)).nan_to_num(0, 0, 0).sum())
            row = q[i].clone()
            row.index_add_(0, at, -p)
            G[i] += wt * T * row
            Gsize[i] += wt * T * q[i]
            Gsize[i].index_add_(0, at, wt * T * p)
        if y is not None and 0 <= y[i] < C:
            loss -= wl * float(ls[i, y[i]])
            size += wl * (float(ls[i, y[i]].abs()) + float(Z[i].abs().max()))
            row = soft[i].clone()
            row[y[i]] -= 1
            G[i] += wl * row
            Gsize[i] += wl * soft[i]
            Gsize[i, y[i]] += wl
    return loss / m, G * scale / m, size / m, Gsize * abs(scale) / m


@pytest.mark.parametrize("type_", ALL)
@pytest.mark.parametrize("at", range(len(DISTILL)))
def test_distill(type_, at):
    g = lib()
    n, C, k, pad, skip = DISTILL[at]
    T = [1.0, 2.0, 4.0, 3.0][(at + ALL.index(type_)) % 4]
    gen = gen_of("distill", type_, at)
    Z = Strided(n, C, type_, pad, skip, normal(gen, (n, C), type_, 2.0))
    if C > 4:
        Z.t[0, 1::3] = float("-inf")                          # classes that cannot be
        Z.t[n - 1, 1::2] = torch.finfo(TYPES[type_]).min
        Z.before = Z.buffer.clone()
    top = torch.stack([torch.randperm(C, generator=gen)[:k] for _ in range(n)]).int()
    t = normal(gen, (n, k), type_, 2.0)
    if C > 4:
        z0 = Z.t.double().cpu()
        for i in (0, n - 1):                                  # the teacher names possible classes there
            top[i] = torch.where(z0[i][top[i].long()] < -1e4, torch.full_like(top[i], -1), top[i])
    if n > 2:
        top[1] = -1                                           # never seen
        top[2, k // 2:] = -1                                  # a short list
        t[2, 0] = float("-inf")
    if n > 4 and k > 1:
        top[3, 0] = C                                         # no class
        top[4, 1] = top[4, 0]                                 # the same class twice
    y = torch.randint(0, C, (n,), generator=gen).int()
    y[::3] = -1
    if C > 4:
        z0 = Z.t.double().cpu()
        for i in (0, n - 1):
            if y[i] >= 0 and z0[i, y[i]] < -1e4:
                y[i] = 0
    if n > 5:
        y[5] = C                                              # no class
    topd = torch.zeros(n, k + 1, dtype=torch.int32, device="cuda")[:, :k].copy_(top)
    td = Strided(n, k, type_, 3, skip, t)
    labels = y.cuda() if at % 4 != 3 else None
    wt, wl, m, scale = 0.7, 0.4, n + 3, 2.5
    G, loss = out(n, C, type_, pad, skip), torch.full((1,), 9.0, device="cuda")
    args = dict(labels=labels, temperature=T, w_teacher=wt, w_label=wl, m=m, grad_scale=scale)
    g.gcn_distill(Z.t, topd, td.t, loss, G.t, **args)
    ref, Gref, size, Gsize = distill64(d64(Z), top.long(), t.double(), y.long() if labels is not None else None, T, wt, wl, m, scale)
    # exponents up to 40 in 32 bits are off by 40 EPS, sums over the row by their additions; the instruction's power of two adds 2^-22 per unit of the argument
    K = (DEPTH + 4 * 40) * EPS
    check(loss, torch.tensor([ref], dtype=torch.float64), K * size + EPS * abs(ref) + 1e-30, "loss")
    check(G.t, Gref, K * Gsize + 4 * EPS * Gsize + UNIT[type_] * Gref.abs() + TINY[type_], "G")
    assert G.outside_is_untouched() and Z.outside_is_untouched()
    again, place = torch.empty(1, device="cuda"), Z.t.clone()
    g.gcn_distill(place, topd, td.t, again, place, **args)
    assert torch.equal(again, loss) and torch.equal(place, G.t), "in place"
    g.gcn_distill(Z.t, topd, td.t, again, **args)
    assert torch.equal(again, loss), "without a gradient"


@pytest.mark.parametrize("C", [23, 700])
def test_distill_gradient_against_differences(C):
    g = lib()
    n, k, T = 13, 6, 2.5
    gen = gen_of("kddiff", C)
    Z, t = normal(gen, (n, C), "f32", 1.5), normal(gen, (n, k), "f32", 1.5)
    top = torch.stack([torch.randperm(C, generator=gen)[:k] for _ in range(n)])
    y = torch.randint(0, C, (n,), generator=gen)
    D = torch.randn(n, C, generator=gen, dtype=torch.float64)

    def value(h):
        z = Z.double() + h * D
        p = torch.softmax(t.double() / T, 1)
        kl = (p * (p.log() - torch.log_softmax(z / T, 1).gather(1, top))).sum()
        return float(0.6 * T * T * kl - 0.4 * torch.log_softmax(z, 1).gather(1, y[:, None]).sum()) / n
    quotient = (value(1e-5) - value(-1e-5)) / 2e-5
    G, loss = torch.empty(n, C, device="cuda"), torch.empty(1, device="cuda")
    g.gcn_distill(Z.cuda(), top.int().cuda(), t.cuda(), loss, G, labels=y.int().cuda(), temperature=T, w_teacher=0.6, w_label=0.4)
    terms = G.double().cpu() * D
    assert abs(float(terms.sum()) - quotient) <= 1000 * EPS * float(terms.abs().sum()) + 1e-8
    assert abs(float(loss) - value(0.0)) <= 1000 * EPS * abs(value(0.0))


def test_distill_rows_without_anything():
    """No list and no label: no loss, a zero gradient, whatever the logits; a row without a possible class is NaN only where it is asked for."""
    g = lib()
    n, C = 5, 20
    Z = torch.randn(n, C, device="cuda")
    Z[2] = float("-inf")
    Z[3, 4] = float("nan")
    top = torch.full((n, 3), -1, dtype=torch.int32, device="cuda")
    t = torch.zeros(n, 3, device="cuda")
    y = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    G, loss = torch.full((n, C), 5.0, device="cuda"), torch.full((1,), 5.0, device="cuda")
    g.gcn_distill(Z, top, t, loss, G, labels=y, w_label=1.0)
    assert float(loss) == 0.0 and bool((G == 0).all())
    y[0], top[1, 0] = 3, 2
    g.gcn_distill(Z, top, t, loss, G, labels=y, w_label=1.0)
    assert math.isfinite(float(loss)) and bool((G[2:] == 0).all()) and bool(torch.isfinite(G[:2]).all())
    top[3, 0] = 1
    g.gcn_distill(Z, top, t, loss, G, labels=y, w_label=1.0)
    assert math.isnan(float(loss)) and bool(torch.isnan(G[3]).all()) and bool(torch.isfinite(G[[0, 1, 2, 4]]).all())


@pytest.mark.parametrize("type_", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1.0, 2.0, 3.0])
@pytest.mark.parametrize("C", [40, 3000, 40000])
def test_distill_nan_makes_its_row_nan(C, T, type_):
    """A few NaN among a row's logits, also where a thread meets nothing else at first; the other rows keep their results."""
    g = lib()
    gen = gen_of("nan", C)
    Z = normal(gen, (3, C), type_).cuda()
    top, t = torch.tensor([[1, C - 1]] * 3, dtype=torch.int32, device="cuda"), normal(gen, (3, 2), type_).cuda()
    y = torch.full((3,), 9, dtype=torch.int32, device="cuda")
    want, G, loss = torch.empty_like(Z), torch.empty_like(Z), torch.empty(1, device="cuda")
    g.gcn_distill(Z, top, t, loss, want, labels=y, temperature=T, w_teacher=0.5, w_label=0.5)
    assert math.isfinite(float(loss))
    Z[1, 16:24] = float("nan")
    g.gcn_distill(Z, top, t, loss, G, labels=y, temperature=T, w_teacher=0.5, w_label=0.5)
    assert math.isnan(float(loss)) and bool(torch.isnan(G[1]).all())
    assert torch.equal(G[0], want[0]) and torch.equal(G[2], want[2])


def test_distill_weight_zero_leaves_a_part_out():
    """A part of weight 0 adds nothing, also where its own loss would be infinite."""
    g = lib()
    n, C = 3, 30
    Z = torch.randn(n, C, device="cuda")
    Z[0, 2] = float("-inf")                                   # impossible, and named by the list and by the label of row 0
    top = torch.full((n, 1), 2, dtype=torch.int32, device="cuda")
    y = torch.full((n,), 2, dtype=torch.int32, device="cuda")
    t = torch.ones(n, 1, device="cuda")
    G, loss = torch.empty(n, C, device="cuda"), torch.empty(1, device="cuda")
    g.gcn_distill(Z, top, t, loss, G, labels=y, w_teacher=1.0, w_label=1.0)
    assert math.isinf(float(loss))
    y[0] = 5
    G1, one = torch.empty_like(G), torch.empty_like(loss)
    g.gcn_distill(Z, top, t, loss, G, labels=y, w_teacher=0.0, w_label=1.0)
    g.gcn_distill(Z, torch.full_like(top, -1), t, one, G1, labels=y, w_teacher=1.0, w_label=1.0)
    assert math.isfinite(float(loss)) and torch.equal(loss, one) and torch.equal(G, G1)
    top[0], y[0] = 5, 2
    g.gcn_distill(Z, top, t, loss, G, labels=y, w_teacher=1.0, w_label=0.0)
    g.gcn_distill(Z, top, t, one, G1, labels=None, w_teacher=1.0, w_label=1.0)
    assert math.isfinite(float(loss)) and torch.equal(loss, one) and torch.equal(G, G1)


def test_distill_refusals():
    g = lib()
    Z, G, t, loss = torch.zeros(4, 8, device="cuda"), torch.zeros(4, 8, device="cuda"), torch.zeros(4, 3, device="cuda"), torch.zeros(1, device="cuda")
    top = torch.zeros(4, 3, dtype=torch.int32, device="cuda")

    def refused(f, text):
        with pytest.raises(g.GcnError) as e:
            f()
        assert e.value.code == -1 and text in str(e.value), str(e.value)
    for T in (0.0, -1.0, float("nan"), float("inf")):
        refused(lambda: g.gcn_distill(Z, top, t, loss, G, temperature=T), "temperature")
    refused(lambda: g.gcn_distill(Z, top, t, loss, G, m=0), "m must")
    refused(lambda: g.gcn_distill(Z[:, :2], top, t, loss, G[:, :2]), "classes")
    refused(lambda: g.gcn_distill(Z[:3], top[:3], t[:3], loss, Z[1:]), "overlaps")
    refused(lambda: g.gcn_distill(Z, top, t, Z.view(-1)[:1], G), "overlaps")
    L = g.lib()
    p = lambda x: x.data_ptr()
    assert L.gcn_distill(4, 8, 0, None, 8, 3, p(top), 3, p(t), 3, None, 1.0, 1.0, 0.0, 4, 1.0, p(loss), p(G), 8, 0) == -1
    assert L.gcn_distill(4, 8, 7, p(Z), 8, 3, p(top), 3, p(t), 3, None, 1.0, 1.0, 0.0, 4, 1.0, p(loss), p(G), 8, 0) == -1
    assert L.gcn_distill(4, 8, 0, p(Z), 7, 3, p(top), 3, p(t), 3, None, 1.0, 1.0, 0.0, 4, 1.0, p(loss), p(G), 8, 0) == -1
    assert L.gcn_distill(0, 8, 0, p(Z), 8, 3, p(top), 3, p(t), 3, None, 1.0, 1.0, 0.0, 4, 1.0, p(loss), p(G), 8, 0) == -1
    assert L.gcn_distill(4, 8, 0, p(Z), 8, 0, p(top), 3, p(t), 3, None, 1.0, 1.0, 0.0, 4, 1.0, p(loss), p(G), 8, 0) == -1


# ---- sizes ----------------------------------------------------------------------------------------------------------
def test_widths_beyond_the_range_are_refused():
    """By every entry point, before anything is launched or read."""
    L, x = lib().lib(), torch.zeros(64, device="cuda")
    p = [x[8 * i:].data_ptr() for i in range(8)]
    far = (1 << 31) - 1
    assert L.gcn_linear_forward(1, 1, (1 << 27) + 1, 0, p[0], far, p[1], far, None, 0, None, 0, 0.0, None, 0, p[2], far, 0) == -2
    assert L.gcn_linear_backward(1, 1, (1 << 27) + 1, 0, p[0], far, p[1], far, None, 0, p[2], far, 0, 0.0, None, 0, None, 0, None, 0, p[3], None, 0, 0) == -2
    for f in ((1 << 26) + 1, far):
        assert L.gcn_block_norm_forward(1, f, 0, 0, 1e-5, p[0], far, None, 0, None, 0, 0, None, None, None, p[1], None, None, 0, p[2], far, None, 0) == -2
        assert L.gcn_block_norm_backward(1, f, 0, 0, None, 0, None, 0, 0, None, None, None, p[0], p[1], far, p[2], None, 0, p[3], far, p[4], far,
                                         None, 0, None, 0, None, None, None, None, None, 0) == -2
    for C in ((1 << 30) + 1, far):
        assert L.gcn_distill(1, C, 0, p[0], far, 1, p[1], 1, p[2], 1, None, 1.0, 1.0, 0.0, 1, 1.0, p[3], None, 0, 0) == -2


@pytest.mark.parametrize("type_", ["f32", "f16"])
def test_linear_backward_of_one_very_wide_row(type_):
    """One row: the bias's gradient is dY act'(Z), and dR is rho dY, both exact for ReLU; more columns than a launch has rows of workgroups."""
    g = lib()
    N = (1 << 25) + 3
    dY, Z = torch.empty(1, N, device="cuda", dtype=TYPES[type_]).normal_(), torch.empty(1, N, device="cuda", dtype=TYPES[type_]).normal_()
    db, dR, dZ = torch.empty(N, device="cuda"), torch.empty_like(dY), torch.empty_like(dY)
    g.gcn_linear_backward(None, None, Z, dY, dZ, dbias=db, dR=dR, act=g.ACT_RELU, rho=0.5)
    assert torch.equal(dZ, dY * (Z > 0)) and torch.equal(db, dZ[0].float()) and torch.equal(dR, (0.5 * dY.float()).to(dY.dtype))


# ---- streams and graphs ---------------------------------------------------------------------------------------------
def test_operators_on_a_stream_of_the_callers_and_in_a_graph():
    """A training step of a block on a side stream, and the same one captured and replayed with new inputs: the eager results bit by bit."""
    g = lib()
    gen = gen_of("graph")
    n, f, C, k = 300, 128, 50, 4
    X, W, W2 = normal(gen, (n, f), "bf16").cuda(), normal(gen, (f, f), "bf16", 0.1).cuda(), normal(gen, (f, C), "bf16", 0.1).cuda()
    w = torch.ones(f, device="cuda")
    top = torch.stack([torch.randperm(C, generator=gen)[:k] for _ in range(n)]).int().cuda()
    t = normal(gen, (n, k), "bf16").cuda()
    e = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt, device="cuda")
    U, Z, Xo, H, logits, G, dH, dX, dU, dZ = e(n, f), e(n, f), e(n, f), e(n, f), e(n, C), e(n, C), e(n, f), e(n, f), e(n, f), e(n, f)
    dW, dW2, dw, stats, loss, db = e(f, f), e(f, C), e(f, dt=torch.float32), e(n, 4, dt=torch.float32), e(1, dt=torch.float32), e(f, dt=torch.float32)

    def step():
        g.gcn_linear_forward(X, W, U, act=g.ACT_GELU, Z=Z)
        g.gcn_block_norm_forward(X, U, Xo, H, w_pre=w, w_post=w, stats=stats)
        g.gcn_linear_forward(H, W2, logits)
        g.gcn_distill(logits, top, t, loss, G, temperature=2.0)
        g.gcn_linear_backward(H, W2, None, G, dX=dH, dW=dW2)
        g.gcn_block_norm_backward(U, Xo, stats, None, dH, dX, dU, w_pre=w, w_post=w, dw_post=dw)
        g.gcn_linear_backward(X, W, Z, dU, dZ, dW=dW, dbias=db, act=g.ACT_GELU)
    outs = (loss, dW, dW2, dw, db, dX, G)
    step()
    torch.cuda.synchronize()
    first = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for o in outs:
            o.zero_()
        step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for round_ in range(3):
        X.copy_(normal(gen, (n, f), "bf16"))
        step()
        torch.cuda.synchronize()
        want = [o.clone() for o in outs]
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs)), round_


def test_linear_offsets_beyond_32_bits():
    """Rows that lie more than 2^32 bytes behind the first."""
    g = lib()
    n, K, N = 3, 24, 40
    ld = (1 << 30) + 8
    buf = torch.empty(2 * ld + 64, dtype=torch.bfloat16, device="cuda")
    gen = gen_of("far")
    X = buf[:].as_strided((n, K), (ld, 1))
    x = normal(gen, (n, K), "bf16").cuda()
    X.copy_(x)
    W = normal(gen, (K, N), "bf16").cuda()
    Y, want = torch.empty(n, N, dtype=torch.bfloat16, device="cuda"), torch.empty(n, N, dtype=torch.bfloat16, device="cuda")
    g.gcn_linear_forward(X, W, Y)
    g.gcn_linear_forward(x, W, want)
    assert torch.equal(Y, want)
    w = torch.ones(K, device="cuda")
    H, hw = torch.empty_like(x), torch.empty_like(x)
    g.gcn_block_norm_forward(X, H=H, w_pre=w)
    g.gcn_block_norm_forward(x, H=hw, w_pre=w)
    assert torch.equal(H, hw)
