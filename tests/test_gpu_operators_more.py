"""The operators of residual networks at the ends of what they take: magnitudes, widths, places of operands, tiles.

Tolerances are derived as in test_gpu_operators.py."""
import math

import pytest

torch = pytest.importorskip("torch")

from test_gpu_operators import ALL, DEPTH, EPS, TINY, TYPES, UNIT, check, gen_of, lib, norm64, normal, unit_gradient64

pytestmark = pytest.mark.gpu


# ---- fp32 products --------------------------------------------------------------------------------------------------
def outer_products(g, x, w):
    """x w^T of two vectors by each of a layer's three products, none of them with a sum: the forward pass, dX and dW."""
    X, W = x.reshape(-1, 1).contiguous().cuda(), w.reshape(1, -1).contiguous().cuda()
    n, N = X.shape[0], W.shape[1]
    Y, dX, dW = (torch.empty(n, N, device="cuda") for _ in range(3))
    g.gcn_linear_forward(X, W, Y)
    g.gcn_linear_backward(None, W.t().contiguous(), None, X, dX=dX)
    g.gcn_linear_backward(X.t().contiguous(), None, None, W, dW=dW)
    return dict(forward=Y, dX=dX, dW=dW)


def test_linear_fp32_products_next_to_the_largest_number():
    """Finite where the product is, though both factors are rounded up on their way, and infinite of the right sign where it is not."""
    g = lib()
    x = torch.full((70,), 1.9999 * 2.0 ** 63)
    x[1::2] *= -1
    x[3], x[4] = 1.0, 2.0 ** 65
    w = torch.full((45,), 1.9999 * 2.0 ** 63)
    w[2::5] *= -1
    ref = x.double()[:, None] * w.double()[None]
    most = torch.finfo(torch.float32).max
    ref = torch.where(ref.abs() > most, ref.sign() * math.inf, ref)
    assert bool(torch.isfinite(ref[0]).all()) and bool(torch.isinf(ref[4]).all())
    for name, got in outer_products(g, x, w).items():
        check(got, ref, 3 * EPS * ref.abs(), name)
        assert torch.equal(got.cpu().sign().double(), ref.sign()), name
    # the same product in a sum of two
    X, W = torch.stack([x, torch.full_like(x, -1.0)], 1), torch.stack([w, torch.full_like(w, 2.0 ** 100)], 0)
    Y = torch.empty(70, 45, device="cuda")
    g.gcn_linear_forward(X.cuda(), W.cuda(), Y)
    fine = torch.isfinite(ref)
    want = torch.where(fine, ref - 2.0 ** 100, ref)
    check(Y, want, 4 * EPS * (ref.abs() + 2.0 ** 100), "sum of two")


def test_linear_fp32_products_whose_parts_are_largest():
    """Mantissas whose second and third parts are as large as they can be: what is left out of their product is 2^-24 of it, and the sum of what is kept is
    rounded as an fp32 product is."""
    g = lib()
    x = 1 + 2.0 ** -8 - 2.0 ** -17 - 2.0 ** -23
    x = torch.full((70,), x) * torch.exp2(torch.arange(70).float() - 35)
    w = torch.full((45,), float(x[35]))
    w[1::2] = -w[1::2]
    assert float(x[35]) == 1 + 2.0 ** -8 - 2.0 ** -17 - 2.0 ** -23
    ref = x.double()[:, None] * w.double()[None]
    for name, got in outer_products(g, x, w).items():
        check(got, ref, 3 * EPS * ref.abs(), name)


# ---- the widest rows ------------------------------------------------------------------------------------------------
def test_block_norm_of_the_widest_row():
    """One row of 2^26 elements through the norms and back.  The root mean square of ones and minus ones is 1 (eps 0) and the gradients are exact."""
    g = lib()
    f = 1 << 26
    X = torch.ones(1, f, dtype=torch.bfloat16, device="cuda")
    X[0, ::3] = -1
    w = torch.full((f,), 2.0, device="cuda")
    H, stats = torch.empty_like(X), torch.empty(1, 4, device="cuda")
    g.gcn_block_norm_forward(X, H=H, w_pre=w, stats=stats, eps=0.0)
    assert torch.equal(H, 2 * X) and stats[0].tolist() == [0, 0, 0, 1]
    # a gradient at right angles to the row: dX = dH w, and the weights' gradient is dH x^
    dH = torch.zeros_like(X)
    dH[0, 0], dH[0, 1], dH[0, f - 2], dH[0, f - 1] = 1.0, 1.0, 3.0, 3.0
    assert float((dH.float() * X.float()).sum()) == 0
    dX, dw, db = torch.empty_like(X), torch.full((f,), 9.0, device="cuda"), torch.full((f,), 9.0, device="cuda")
    g.gcn_block_norm_backward(None, X, stats, None, dH, dX, w_pre=w, dw_pre=dw, db_pre=db)
    assert torch.equal(dX, 2 * dH) and torch.equal(dw, (dH * X)[0].float()) and torch.equal(db, dH[0].float())


def test_gradient_of_a_gate_in_place_of_a_row_of_one_element():
    """Rows of one element: the gate is as wide as they are, so its gradient may take the place of any of the row's operands."""
    g = lib()
    n = 5
    gen = gen_of("one")
    u, a, xo, c, d = (normal(gen, (n, 1), "f32").cuda() for _ in range(5))
    w = torch.tensor([1.5], device="cuda")
    stats = torch.rand(n, 4, generator=gen).cuda() + 0.5
    e = lambda: torch.empty(n, 1, device="cuda")
    want = [e(), e(), e()]
    g.gcn_block_norm_backward(u, xo, stats, c, d, *want[:2], w_pre=w, w_post=w, A=a, dA=want[2], kind=g.NORM_LAYER)
    for name in ("U", "A", "Xout", "dXout", "dH"):
        o = dict(U=u.clone(), A=a.clone(), Xout=xo.clone(), dXout=c.clone(), dH=d.clone())
        dX, dU = e(), e()
        g.gcn_block_norm_backward(o["U"], o["Xout"], stats, o["dXout"], o["dH"], dX, dU, w_pre=w, w_post=w, A=o["A"], dA=o[name], kind=g.NORM_LAYER)
        assert torch.equal(dX, want[0]) and torch.equal(dU, want[1]) and torch.equal(o[name], want[2]), name


# ---- rows longer than registers hold, and shorter than a lane's elements --------------------------------------------
@pytest.mark.parametrize("type_", ALL)
@pytest.mark.parametrize("n,f,gate,layer", [(70, 9001, "full", True), (133, 8200, "row", False), (37, 16384, None, True), (5000, 3, "row", True),
                                            (3001, 2, "full", False), (257, 1, "row", False)])
def test_block_norm_backward_of_many_rows(type_, n, f, gate, layer):
    """Rows in several shares: every gradient against the formula in 64 bits, and the vectors' the same bits in every call."""
    g = lib()
    gen = gen_of("long", type_, n, f)
    columns = {"full": f, "row": 1, None: 0}[gate]
    U, Xo, C, D = (normal(gen, (n, f), type_, s).cuda() for s in (2.0, 1.3, 1.0, 1.0))
    A = normal(gen, (n, columns), type_).cuda() if gate else None
    vec = lambda c: (c + 0.2 * torch.randn(f, generator=gen, dtype=torch.float64)).float().cuda()
    scale, wp, w = vec(0.3), vec(1.0), vec(1.0)
    bp = vec(0.0) if layer else None
    xo, u, c, d, sc, w2, wp2 = (t.double() for t in (Xo, U, C, D, scale, w, wp))
    stats64 = torch.zeros(n, 4, dtype=torch.float64, device="cuda")
    _, stats64[:, 0:1], stats64[:, 1:2], _ = norm64(u, wp2, None, layer)
    _, stats64[:, 2:3], stats64[:, 3:4], _ = norm64(xo, w2, None, layer)
    stats = stats64.float()
    um, ur, xm, xr = stats.double().split(1, dim=1)
    e = lambda *s: torch.full(s, 7.0, dtype=TYPES[type_], device="cuda")
    v = lambda: torch.full((f,), 7.0, device="cuda")
    out = dict(dX=e(n, f), dU=e(n, f), dA=e(n, columns) if gate else None, dscale=v(), dw_post=v(), db_post=v() if layer else None, dw_pre=v(), db_pre=v())
    common = dict(w_pre=w, A=A, scale=scale, w_post=wp, b_post=bp, kind=g.NORM_LAYER if layer else g.NORM_RMS)
    g.gcn_block_norm_backward(U, Xo, stats, C, D, **out, **common)
    K, unit, tiny = 4 * DEPTH * EPS, UNIT[type_], TINY[type_]
    xhat, xsize = (xo - xm) * xr, (xo.abs() + xm.abs()) * xr
    dx = c + unit_gradient64(d * w2, xhat, xr, layer)[0]
    size = c.abs() + unit_gradient64((d * w2).abs(), xsize, xr, True)[1]
    s = torch.sigmoid(A.double()) if gate else torch.ones(n, 1, dtype=torch.float64, device="cuda")
    b = bp.double() if layer else 0 * sc
    uhat, usize = (u - um) * ur, (u.abs() + um.abs()) * ur
    val, vsize = uhat * wp2 + b, usize * wp2.abs() + b.abs()
    dv, dvsize = dx * sc * s, size * sc.abs() * s
    du = unit_gradient64(dv * wp2, uhat, ur, layer)[0]
    dusize = unit_gradient64(dvsize * wp2.abs(), usize, ur, True)[1]
    check(out["dX"], dx.cpu(), (K * size + unit * dx.abs() + tiny).cpu(), "dX")
    check(out["dU"], du.cpu(), (K * dusize + unit * du.abs() + tiny).cpu(), "dU")
    if gate:
        da, dasize = dx * sc * val * s * (1 - s), size * sc.abs() * vsize * s
        if columns != f:
            da, dasize = da.sum(1, keepdim=True), dasize.sum(1, keepdim=True)
        check(out["dA"], da.cpu(), (K * dasize + unit * da.abs() + tiny).cpu(), "dA")
    KV = K + (n + 2) * EPS
    sums = dict(dscale=(dx * s * val, size * s * vsize), dw_post=(dv * uhat, dvsize * usize), db_post=(dv, dvsize), dw_pre=(d * xhat, d.abs() * xsize),
                db_pre=(d, d.abs()))
    for name, (terms, sizes) in sums.items():
        if out[name] is not None:
            check(out[name], terms.sum(0).cpu(), (KV * sizes.sum(0) + 1e-37).cpu(), name)
    # again, in place of the inputs
    again = {k: torch.empty_like(t) for k, t in out.items() if t is not None and t.dim() == 1}
    place = dict(dX=U.clone(), dU=C.clone(), dA=A.clone() if gate else None)
    g.gcn_block_norm_backward(place["dX"], Xo, stats, place["dU"], D, **place, **again, **dict(common, A=place["dA"]))
    assert all(torch.equal(t, out[k]) for k, t in {**again, **place}.items() if t is not None)


def test_scratch_of_a_norm_s_gradients_is_bounded():
    """256 rows of 2^18 elements: the call keeps some tens of megabytes of partial sums, not a copy of its operands in fp32."""
    g = lib()
    n, f = 256, 1 << 18
    e = lambda: torch.zeros(n, f, dtype=torch.bfloat16, device="cuda")
    U, Xo, D, stats = e(), e(), e(), torch.ones(n, 4, device="cuda")
    v = [torch.ones(f, device="cuda") for _ in range(6)]
    torch.cuda.synchronize()
    g.gcn_scratch_release()
    before = torch.cuda.mem_get_info()[0]
    g.gcn_block_norm_backward(U, Xo, stats, None, D, w_pre=v[0], w_post=v[1], dscale=v[2], dw_post=v[3], db_post=v[4], dw_pre=v[5], kind=g.NORM_LAYER)
    torch.cuda.synchronize()
    assert before - torch.cuda.mem_get_info()[0] < (64 << 20)
    assert all(bool((t == 0).all()) for t in v[2:])


# ---- operands side by side ------------------------------------------------------------------------------------------
def halves(n, left, right, dtype, mark=3.0):
    """Two matrices whose rows take turns in one buffer."""
    both = torch.full((n, left + right), mark, dtype=dtype, device="cuda")
    return both[:, :left], both[:, left:]


@pytest.mark.parametrize("type_", ALL)
@pytest.mark.parametrize("n,K,N", [(5, 48, 40), (200, 65, 130)])
def test_linear_operands_side_by_side(type_, n, K, N):
    """Y beside Z, Y beside X, and the gradients beside what they are made of: the results of matrices by themselves."""
    g = lib()
    dt = TYPES[type_]
    gen = gen_of("beside", type_, n)
    x, W, dy = normal(gen, (n, K), type_).cuda(), normal(gen, (K, N), type_, K ** -0.5).cuda(), normal(gen, (n, N), type_).cuda()
    e = lambda *s: torch.empty(*s, dtype=dt, device="cuda")
    y0, z0 = e(n, N), e(n, N)
    g.gcn_linear_forward(x, W, y0, act=g.ACT_SILU, Z=z0)
    Y, Z = halves(n, N, N, dt)
    g.gcn_linear_forward(x, W, Y, act=g.ACT_SILU, Z=Z)
    assert torch.equal(Y, y0) and torch.equal(Z, z0)
    X, Y = halves(n, K, N, dt)
    X.copy_(x)
    g.gcn_linear_forward(X, W, Y, act=g.ACT_SILU)
    assert torch.equal(Y, y0) and torch.equal(X, x)
    dz0, dx0, dw0 = e(n, N), e(n, K), e(K, N)
    g.gcn_linear_backward(x, W, z0, dy, dz0, dX=dx0, dW=dw0, act=g.ACT_SILU)
    Z, dZ = halves(n, N, N, dt)
    Z.copy_(z0)
    X, dX = halves(n, K, K, dt)
    X.copy_(x)
    V, dW = halves(K, N, N, dt)
    V.copy_(W)
    g.gcn_linear_backward(X, V, Z, dy, dZ, dX=dX, dW=dW, act=g.ACT_SILU)
    assert torch.equal(dZ, dz0) and torch.equal(dX, dx0) and torch.equal(dW, dw0)
    assert torch.equal(Z, z0) and torch.equal(X, x) and torch.equal(V, W)
    # one element in common, at the end of a row and at the start of the next
    wide = torch.zeros(n, 2 * N, dtype=dt, device="cuda")
    for at in (N - 1, 1):
        with pytest.raises(g.GcnError, match="overlaps"):
            g.gcn_linear_forward(x, W, wide[:, :N], Z=wide[:, at:at + N])


@pytest.mark.parametrize("type_", ALL)
@pytest.mark.parametrize("f", [5, 130, 9001])
def test_block_norm_operands_side_by_side(type_, f):
    """U and A from one wide product, their gradients likewise, X' beside H."""
    g = lib()
    dt, n = TYPES[type_], 6
    gen = gen_of("besidenorm", type_, f)
    x, u, a, c, d = (normal(gen, (n, f), type_).cuda() for _ in range(5))
    w = torch.ones(f, device="cuda")
    e = lambda: torch.empty(n, f, dtype=dt, device="cuda")
    xo, h, dx, du, da, stats = e(), e(), e(), e(), e(), torch.empty(n, 4, device="cuda")
    g.gcn_block_norm_forward(x, u, xo, h, w_pre=w, w_post=w, A=a, stats=stats)
    g.gcn_block_norm_backward(u, xo, stats, c, d, dx, du, w_pre=w, w_post=w, A=a, dA=da)
    (U, A), (Xo, H), (dU, dA) = (halves(n, f, f, dt) for _ in range(3))
    U.copy_(u), A.copy_(a)
    g.gcn_block_norm_forward(x, U, Xo, H, w_pre=w, w_post=w, A=A)
    assert torch.equal(Xo, xo) and torch.equal(H, h)
    dX = e()
    g.gcn_block_norm_backward(U, Xo, stats, c, d, dX, dU, w_pre=w, w_post=w, A=A, dA=dA)
    assert torch.equal(dX, dx) and torch.equal(dU, du) and torch.equal(dA, da)
    g.gcn_block_norm_backward(U, Xo, stats, c, d, dX, U, w_pre=w, w_post=w, A=A, dA=A)      # each in the place of its own operand
    assert torch.equal(U, du) and torch.equal(A, da)
    with pytest.raises(g.GcnError, match="overlaps"):
        wide = torch.zeros(n, 2 * f, dtype=dt, device="cuda")
        g.gcn_block_norm_forward(x, u, wide[:, :f], wide[:, f - 1:2 * f - 1], w_pre=w)


def test_one_row_in_place_whatever_its_leading_dimension():
    """A single row has no other: its place is its address and width."""
    g = lib()
    f = 40
    x = torch.randn(1, f, device="cuda")
    w, want, place = torch.ones(f, device="cuda"), torch.empty_like(x), x.clone()
    g.gcn_block_norm_forward(x, H=want, w_pre=w)
    L, p = g.lib(), place.data_ptr()
    rc = L.gcn_block_norm_forward(1, f, g.F32, g.NORM_RMS, 1e-5, p, f, None, 0, None, 0, 0, None, None, None, w.data_ptr(), None, None, 0, p, 2 * f, None,
                                  g.binding._now())
    assert rc == 0 and torch.equal(place, want)


@pytest.mark.parametrize("type_", ALL)
@pytest.mark.parametrize("C", [41, 700, 20001])
def test_distill_gradient_beside_the_logits(type_, C):
    g = lib()
    dt, n, k = TYPES[type_], 5, 3
    gen = gen_of("besidekd", type_, C)
    z, t = normal(gen, (n, C), type_).cuda(), normal(gen, (n, k), type_).cuda()
    top = torch.stack([torch.randperm(C, generator=gen)[:k] for _ in range(n)]).int().cuda()
    g0, loss0, loss = torch.empty_like(z), torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    g.gcn_distill(z, top, t, loss0, g0)
    Z, G = halves(n, C, C, dt)
    Z.copy_(z)
    g.gcn_distill(Z, top, t, loss, G)
    assert torch.equal(G, g0) and torch.equal(loss, loss0) and torch.equal(Z, z)


# ---- exponentials of fp32 elements ----------------------------------------------------------------------------------
# A power of e off by 2 units in the last place (4 EPS), 1 added, a reciprocal off by one (2 EPS), and up to three products.
POWERS = 12 * EPS


def far():
    return torch.cat([torch.linspace(-85, 85, 3401), torch.tensor([0.0, -0.5, 1e-6, -1e-6])])


def test_silu_of_fp32_far_from_zero():
    """The activation relative to itself; its slope, whose two terms cancel where it is 0, relative to them."""
    g = lib()
    z = far()
    n = z.numel()
    X, W = z.reshape(n, 1).cuda(), torch.ones(1, 1, device="cuda")
    Y = torch.empty(n, 1, device="cuda")
    g.gcn_linear_forward(X, W, Y, act=g.ACT_SILU)
    s = torch.sigmoid(z.double())
    check(Y[:, 0], z.double() * s, POWERS * (z.double() * s).abs() + 1e-37, "silu")
    few = torch.empty(5, 1, device="cuda")
    g.gcn_linear_forward(X[:5], W, few, act=g.ACT_SILU)
    assert torch.equal(few, Y[:5])
    dZ = torch.empty(n, 1, device="cuda")
    g.gcn_linear_backward(None, None, X, torch.ones(n, 1, device="cuda"), dZ, act=g.ACT_SILU)
    # (1 - s) is off by what s is off, relative to 1
    check(dZ[:, 0], s * (1 + z.double() * (1 - s)), 2 * POWERS * s * (1 + z.double().abs()) + 1e-37, "slope")


@pytest.mark.parametrize("f", [3405, 20430])
@pytest.mark.parametrize("per_row", [False, True])
def test_gate_of_fp32_far_from_zero(f, per_row):
    """X' = sigmoid(A) for U = 1 and X = 0, in rows of registers and in longer ones; dU = sigmoid(A) dX'."""
    g = lib()
    a = far().repeat(f // 3405)
    n = 7 if per_row else 1
    A = a[::500][:n].reshape(n, 1) if per_row else a.reshape(1, f)
    X, U, Xo = torch.zeros(n, f, device="cuda"), torch.ones(n, f, device="cuda"), torch.empty(n, f, device="cuda")
    g.gcn_block_norm_forward(X, U, Xo, A=A.cuda())
    s = torch.sigmoid(A.double()).expand(n, f)
    check(Xo, s, POWERS * s, "gate")
    dU = torch.empty(n, f, device="cuda")
    g.gcn_block_norm_backward(U, None, torch.zeros(n, 4, device="cuda"), U, None, None, dU, A=A.cuda())
    check(dU, s, POWERS * s, "dU")


@pytest.mark.parametrize("T", [1.0, 2.0, 3.0, 4.0])
@pytest.mark.parametrize("C", [41, 700, 20001])
def test_distill_of_fp32_logits_far_apart(C, T):
    """The gradient of classes far below the largest, relative to itself: the exponential is off by 2^-23 for each unit of its exponent, and its constant, which 1 / T and
    log2(e) are rounded into, by as much again at the most."""
    g = lib()
    d = torch.linspace(0, 80, C)
    Z = (-d * T).reshape(1, C)
    top, t = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.zeros(1, 1, device="cuda")
    G, loss = torch.empty(1, C, device="cuda"), torch.empty(1, device="cuda")
    g.gcn_distill(Z.cuda(), top, t, loss, G, temperature=T)
    z = Z.double() / T
    q = torch.softmax(z, 1)
    # the sum of the row is off by its additions; the first column's gradient is q - 1
    tol = T * (POWERS + 40 * EPS + 4 * EPS * z.abs()) * q
    tol[0, 0] += 4 * EPS * T
    ref = T * q
    ref[0, 0] -= T
    check(G, ref, tol, "G")


# ---- temperatures ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("T", [2.0 ** -126, 1e-25, 1e-12, 1e12])
def test_distill_at_the_ends_of_the_temperatures(T):
    """One entry, one below the row's largest logit of two: the loss is T^2 log(1 + e^(1/T)), or T at low temperatures, and T (q - p) the gradient."""
    g = lib()
    Z, t = torch.tensor([[0.0, 1.0]], device="cuda"), torch.zeros(1, 1, device="cuda")
    top = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    G, loss = torch.empty(1, 2, device="cuda"), torch.empty(1, device="cuda")
    T = float(torch.tensor(T))                                 # as the call takes it
    g.gcn_distill(Z, top, t, loss, G, temperature=T)
    low = 1 / T > 80
    want = T if low else T * T * math.log1p(math.exp(1 / T))
    assert abs(float(loss) - want) <= 8 * EPS * want
    q = 1.0 if low else 1 / (1 + math.exp(-1 / T))
    for got, ref in zip(G[0].tolist(), (-T * q, T * q)):
        assert abs(got - ref) <= 16 * EPS * T + 2.0 ** -149


def test_distill_refuses_temperatures_without_an_inverse():
    g = lib()
    Z, t, loss = torch.zeros(1, 2, device="cuda"), torch.zeros(1, 1, device="cuda"), torch.zeros(1, device="cuda")
    top = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    with pytest.raises(g.GcnError, match="temperatures"):
        g.gcn_distill(Z, top, t, loss, temperature=2.0 ** -140)
