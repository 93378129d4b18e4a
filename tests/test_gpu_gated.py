"""Gated blocks, checkpoints in 8 bits and weights in 4 bits against plain implementations in 64 bits, through the C ABI.

Codes, scales and what they stand for are equal; other tolerances are derived as in test_gpu_operators.py: K terms summed in 32 bits are off by K 2^-24 times the
sum of their absolute values at most, a rounding to a type by half a unit, elementary functions by a few 2^-24."""
import math

import pytest

torch = pytest.importorskip("torch")

import held
from test_gpu_operators import ACTS, ALL, EPS, SLOPE_MOST, TINY, TYPES, UNIT, Strided, act64, check, code, gen_of, lib, normal, out, slope64

pytestmark = pytest.mark.gpu


class Bytes:
    """Codes of a checkpoint, n x f int8 in rows `pad` apart, `skip` in front, and its scales likewise; marked outside."""

    def __init__(self, n, f, pad=0, skip=0):
        self.n, self.f, self.groups = n, f, -(-f // held.GROUP)
        self.cb = torch.full((skip + n * (f + pad) + 64,), 77, dtype=torch.int8, device="cuda")
        self.sb = torch.full((skip + n * (self.groups + pad) + 64,), 3.0, dtype=torch.bfloat16, device="cuda")
        self.codes = self.cb[skip:skip + n * (f + pad)].view(n, f + pad)[:, :f]
        self.scales = self.sb[skip:skip + n * (self.groups + pad)].view(n, self.groups + pad)[:, :self.groups]

    def pair(self):
        return self.codes, self.scales

    def outside_is_untouched(self):
        c, s = self.cb.clone(), self.sb.clone()
        self.codes.fill_(77)
        self.scales.fill_(3.0)
        fine = bool((self.cb == 77).all()) and bool((self.sb == 3.0).all())
        self.cb.copy_(c)
        self.sb.copy_(s)
        return fine

    def values(self, dtype):
        return held.unpack64(self.codes.cpu(), self.scales.cpu(), dtype)


def kept(x, type_, pad, skip):
    """x as a checkpoint made on the CPU, and the values that it stands for."""
    c, s = held.pack64(x, type_)
    b = Bytes(*x.shape, pad, skip)
    b.codes.copy_(c.to(torch.int8))
    b.scales.copy_(s.bfloat16())
    return b, b.values(TYPES[type_])


def weights(w, group, type_, pad, skip):
    """Weights in 4 bits made on the CPU, in rows `pad` apart (words and scales outside hold what would be seen), and what they stand for."""
    code, s = held.pack4_64(w, group, type_)
    words = held.words4(code)
    Q = torch.full((skip + words.shape[0] * (words.shape[1] + pad) + 64,), 0x77777777, dtype=torch.int32, device="cuda")
    S = torch.full((skip + s.shape[0] * (s.shape[1] + pad) + 64,), float("nan"), dtype=torch.bfloat16, device="cuda")
    q = Q[skip:skip + words.shape[0] * (words.shape[1] + pad)].view(words.shape[0], -1)[:, :words.shape[1]]
    t = S[skip:skip + s.shape[0] * (s.shape[1] + pad)].view(s.shape[0], -1)[:, :s.shape[1]]
    q.copy_(words)
    t.copy_(s.bfloat16())
    return q, t, held.unpack4_64(code, s, group)


# ---- checkpoints: stored and restored -------------------------------------------------------------------------------
ROWS = [(1, 1, 0, 0), (1, 64, 0, 0), (3, 65, 0, 1), (5, 63, 3, 0), (4, 7, 1, 3), (2, 8, 0, 0), (9, 3, 0, 0), (257, 602, 0, 0), (1000, 128, 0, 0), (17, 1000, 5, 2),
        (2, 8195, 0, 0), (4099, 72, 8, 8), (70001, 2, 0, 0), (3, 70001, 0, 0)]


def varied(gen, shape, type_):
    """Numbers of very different sizes, columns and rows of their own; some rows zero."""
    n, f = shape
    x = torch.randn(shape, generator=gen, dtype=torch.float64)
    x *= torch.exp2(torch.randint(-6, 7, (1, f), generator=gen).double()) * torch.exp2(torch.randint(-4, 5, (n, 1), generator=gen).double())
    x[torch.rand(n, generator=gen) < 0.1] = 0
    return x.to(TYPES[type_])


@pytest.mark.parametrize("type_", ALL)
@pytest.mark.parametrize("at", range(len(ROWS)))
def test_checkpoint_is_the_nearest(type_, at):
    g = lib()
    n, f, pad, skip = ROWS[at]
    X = Strided(n, f, type_, pad, skip, varied(gen_of("pack", type_, at), (n, f), type_))
    b = Bytes(n, f, pad, skip)
    g.gcn_checkpoint_pack(X.t, b.codes, b.scales)
    c, s = held.pack64(X.t.cpu(), type_)
    assert torch.equal(b.scales.double().cpu(), s)
    assert torch.equal(b.codes.double().cpu(), c)
    assert b.outside_is_untouched()
    back = out(n, f, type_, pad, skip)
    g.gcn_checkpoint_unpack(b.codes, b.scales, back.t)
    assert torch.equal(back.t.double().cpu(), b.values(TYPES[type_])) and back.outside_is_untouched()


@pytest.mark.parametrize("type_", ALL)
def test_checkpoint_of_ties_and_neighbours(type_):
    """Every middle between two codes and the numbers of the type on both sides of it, for scales of all mantissas."""
    g = lib()
    dt = TYPES[type_]
    rows = []
    for mantissa in range(128, 256):
        s = mantissa / 128.0
        x = torch.cat([torch.tensor([127 * s]), (torch.arange(-126, 127).double() + 0.5) * s]).to(dt)
        bits = x.view(torch.int32 if dt == torch.float32 else torch.int16)
        for step in (-1, 0, 1):
            y = (bits + step).view(dt)
            y[0] = float(torch.tensor(127 * s).to(dt))                # (the largest of the first group decides its scale)
            row = torch.nn.functional.pad(y, (0, -y.numel() % 63)).view(-1, 63)
            rows.append(torch.cat([y[:1].expand(row.shape[0], 1), row], 1).reshape(-1))
    X = torch.stack(rows)
    b = Bytes(*X.shape)
    g.gcn_checkpoint_pack(X.cuda(), b.codes, b.scales)
    c, s = held.pack64(X, type_)
    assert torch.equal(b.scales.double().cpu(), s) and torch.equal(b.codes.double().cpu(), c)
    if type_ == "f32":                                                # middles are numbers of the type: ties were among them
        q = held.grouped(X.double(), held.GROUP) / s[:, :, None]
        assert int((q - q.floor() == 0.5).sum()) > 10000


@pytest.mark.parametrize("type_", ALL)
def test_checkpoint_at_the_ends_of_the_type(type_):
    """The largest numbers, the smallest, and groups that are not finite."""
    g = lib()
    dt = TYPES[type_]
    info = torch.finfo(dt)
    x = torch.zeros(8, 200, dtype=dt)
    x[0, ::3], x[0, 1::3] = info.max, -info.max / 2
    x[1, 5] = float("nan")
    x[2, 70], x[2, 150] = float("inf"), -float("inf")
    x[3, :] = 1.0
    x[4, ::2] = info.tiny
    x[5, ::2], x[5, 1] = info.smallest_normal * info.eps, info.smallest_normal * 3
    x[6, :100] = -0.0
    x[7, 199] = info.max
    b = Bytes(8, 200)
    g.gcn_checkpoint_pack(x.cuda(), b.codes, b.scales)
    c, s = held.pack64(x, type_)
    fine = torch.isfinite(s)
    assert torch.equal(torch.isnan(b.scales.cpu()), ~fine)
    assert torch.equal(b.scales.double().cpu()[fine], s[fine])
    ok = fine.repeat_interleave(held.GROUP, 1)[:, :200]
    assert torch.equal(b.codes.double().cpu()[ok], c[ok])
    back = torch.empty_like(x, device="cuda")
    g.gcn_checkpoint_unpack(b.codes, b.scales, back)
    assert torch.equal(torch.isnan(back.cpu()), ~ok) and bool(torch.isfinite(back.cpu()[ok]).all())
    assert torch.equal(back.double().cpu()[ok], b.values(dt)[ok])


# ---- weights in 4 bits: laid out and read back ----------------------------------------------------------------------
LAYOUTS = [(1, 1, 32, 0, 0), (8, 5, 32, 0, 0), (31, 64, 32, 3, 1), (64, 300, 64, 0, 0), (65, 7, 64, 0, 0), (127, 129, 128, 1, 0), (1000, 41, 128, 0, 0), (4099, 96, 64, 8, 8), (16, 4097, 32, 0, 0)]


@pytest.mark.parametrize("type_", ALL)
@pytest.mark.parametrize("at", range(len(LAYOUTS)))
def test_weights_are_the_nearest(type_, at):
    g = lib()
    K, cols, group, pad, skip = LAYOUTS[at]
    W = Strided(K, cols, type_, pad, skip, varied(gen_of("pack4", type_, at), (K, cols), type_))
    rows, groups = -(-K // 8), -(-K // group)
    Qb = torch.full((skip + rows * (cols + pad) + 64,), 77, dtype=torch.int32, device="cuda")
    Sb = torch.full((skip + groups * (cols + pad) + 64,), 3.0, dtype=torch.bfloat16, device="cuda")
    Q = Qb[skip:skip + rows * (cols + pad)].view(rows, -1)[:, :cols]
    S = Sb[skip:skip + groups * (cols + pad)].view(groups, -1)[:, :cols]
    g.gcn_linear4_pack(W.t, Q, S, group=group)
    c, s = held.pack4_64(W.t.cpu(), group, type_)
    assert torch.equal(S.double().cpu(), s)
    assert torch.equal(Q.cpu(), held.words4(c))
    back = out(K, cols, type_, pad, skip)
    g.gcn_linear4_unpack(Q, S, back.t, group=group)
    assert torch.equal(back.t.double().cpu(), held.unpack4_64(c, s, group).to(TYPES[type_]).double()) and back.outside_is_untouched()
    Q.fill_(77)
    S.fill_(3.0)
    assert bool((Qb == 77).all()) and bool((Sb == 3.0).all())


@pytest.mark.parametrize("type_", ALL)
def test_weights_of_ties_and_at_the_ends(type_):
    g = lib()
    dt = TYPES[type_]
    info = torch.finfo(dt)
    columns = []
    for mantissa in range(128, 256):
        s = mantissa / 128.0
        x = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, 0.0]).double() * s
        x = x.to(dt)
        bits = x.view(torch.int32 if dt == torch.float32 else torch.int16)
        for step in (-1, 0, 1):
            y = (bits + step).view(dt)
            y[0], y[15] = x[0], -0.0
            columns.append(torch.cat([y, y]))
    special = torch.zeros(9, 32, dtype=dt)
    special[0, 3] = float("nan")
    special[1, 31] = -float("inf")
    special[2, ::2] = info.max
    special[3, :] = info.tiny
    special[4, 1] = -info.smallest_normal * info.eps
    special[5, 0] = -info.max
    W = torch.cat([torch.stack(columns), special]).t().contiguous()
    cols = W.shape[1]
    Q, S = torch.empty(4, cols, dtype=torch.int32, device="cuda"), torch.empty(1, cols, dtype=torch.bfloat16, device="cuda")
    g.gcn_linear4_pack(W.cuda(), Q, S, group=32)
    c, s = held.pack4_64(W, 32, type_)
    fine = torch.isfinite(s[0])
    assert torch.equal(torch.isnan(S[0].cpu()), ~fine) and int((~fine).sum()) == 2
    assert torch.equal(S[0].double().cpu()[fine], s[0][fine]) and torch.equal(Q.cpu()[:, fine], held.words4(c)[:, fine])
    back = torch.empty(32, cols, dtype=dt, device="cuda")
    g.gcn_linear4_unpack(Q, S, back, group=32)
    assert bool(torch.isnan(back[:, ~fine]).all()) and bool(torch.isfinite(back[:, fine]).all())


# ---- gated blocks ---------------------------------------------------------------------------------------------------
# n, f_in, f_out, padding between rows, elements in front
GATED = [(1, 1, 1, 0, 0), (1, 64, 64, 0, 0), (1, 1000, 300, 0, 0), (2, 4096, 40, 8, 0), (3, 5, 7, 0, 1), (16, 512, 1024, 0, 0), (17, 33, 65, 3, 0), (32, 160, 96, 0, 8), (33, 160, 96, 0, 8),
         (64, 64, 64, 0, 0), (65, 128, 129, 0, 0), (130, 602, 41, 0, 0), (257, 96, 304, 16, 0), (1000, 37, 8, 0, 0), (2049, 72, 808, 0, 0), (2049, 71, 801, 1, 1),
         (4099, 136, 2048, 0, 0), (20001, 48, 24, 0, 0), (9, 3000, 17, 0, 0), (8, 24, 20000, 0, 0), (5003, 9, 5, 0, 0), (3001, 16, 1, 2, 1), (700, 30, 200, 0, 0),
         (1201, 8, 513, 0, 0), (515, 8, 300, 0, 0), (260, 24, 720, 4, 1)]


def product_off(x, w, b):
    """z = x w + b in 64 bits and how far its sum in 32 may be off."""
    z = x @ w + (0 if b is None else b)
    return z, (x.shape[1] + 2) * EPS * (x.abs() @ w.abs() + (0 if b is None else b.abs()))


def gate64(z, off, act):
    """act(zg) zu and how far it may be off, for z off by `off`."""
    m = z.shape[1] // 2
    zg, zu, og, ou = z[:, :m], z[:, m:], off[:, :m], off[:, m:]
    a = act64(zg, act)
    a_off = SLOPE_MOST * og + 8 * EPS * (zg.abs() + 1e-30)
    return a * zu, a_off * (zu.abs() + ou) + a.abs() * ou + 2 * EPS * (a * zu).abs()


@pytest.mark.parametrize("type_", ALL)
@pytest.mark.parametrize("at", range(len(GATED)))
def test_gated_forward(type_, at):
    g = lib()
    n, K, N, pad, skip = GATED[at]
    act, keep = ACTS[(at + ALL.index(type_)) % 4], at % 3 != 1
    gen = gen_of("gated", type_, at)
    X = Strided(n, K, type_, pad, skip, normal(gen, (n, K), type_))
    W = Strided(K, 2 * N, type_, pad, skip, normal(gen, (K, 2 * N), type_, K ** -0.5))
    b = normal(gen, (2 * N,), "f32").cuda() if at % 4 else None
    H, Z = out(n, N, type_, pad, skip), out(n, 2 * N, type_, pad, skip)
    g.gcn_gated_forward(X.t, W.t, H.t, bias=b, act=code(g, act), Z=Z.t if keep else None)
    z, off = product_off(X.t.double().cpu(), W.t.double().cpu(), None if b is None else b.double().cpu())
    h, h_off = gate64(z, off, act)
    u = UNIT[type_]
    check(H.t, h, h_off + u * (h.abs() + h_off) + TINY[type_], "H")
    if keep:
        check(Z.t, z, off + u * (z.abs() + off) + TINY[type_], "Z")
    assert H.outside_is_untouched() and Z.outside_is_untouched()
    again = out(n, N, type_, pad, skip)
    g.gcn_gated_forward(X.t, W.t, again.t, bias=b, act=code(g, act), Z=None if keep else Z.t)
    assert torch.equal(again.t, H.t), "the same call gives other bits"


def gated_back64(x, w, z, dh, act, type_):
    """dZ, H, dX, dW, dbias in 64 bits, each with how far it may be off before its own rounding."""
    n, m, u = z.shape[0], z.shape[1] // 2, UNIT[type_]
    zg, zu = z[:, :m], z[:, m:]
    a, sl = act64(zg, act), slope64(zg, act)
    dz = torch.cat([dh * zu * sl, dh * a], 1)
    near = torch.cat([10 * EPS * (zg.abs() + 2) * (dh * zu).abs(), 10 * EPS * (zg.abs() + 1e-30) * dh.abs()], 1)
    dz_off = near + u * (dz.abs() + near) + TINY[type_]
    size = dz.abs() + dz_off
    return dict(H=(a * zu, 10 * EPS * zg.abs() * zu.abs()), dZ=(dz, near),
                dX=(dz @ w.t(), dz_off @ w.t().abs() + (2 * m + 2) * EPS * (size @ w.t().abs())),
                dW=(x.t() @ dz, x.t().abs() @ dz_off + (n + 2) * EPS * (x.t().abs() @ size)),
                dbias=(dz.sum(0), near.sum(0) + (n + 2) * EPS * (dz.abs() + near).sum(0)))


@pytest.mark.parametrize("which", ["elements", "checkpoints", "mixed"])
@pytest.mark.parametrize("type_", ALL)
@pytest.mark.parametrize("at", range(len(GATED)))
def test_gated_backward(type_, at, which):
    g = lib()
    n, K, N, pad, skip = GATED[at]
    act = ACTS[(at + 1 + ALL.index(type_)) % 4]
    gen = gen_of("gated back", type_, at)
    x, z = normal(gen, (n, K), type_), normal(gen, (n, 2 * N), type_)
    W = Strided(K, 2 * N, type_, pad, skip, normal(gen, (K, 2 * N), type_, K ** -0.5))
    dH = Strided(n, N, type_, pad, skip, normal(gen, (n, N), type_))
    if which == "elements":
        X, Z = Strided(n, K, type_, pad, skip, x).t, Strided(n, 2 * N, type_, pad, skip, z).t
        x, z = x.double(), z.double()
    else:
        bx, x8 = kept(x, type_, pad, skip)
        bz, z8 = kept(z, type_, pad, skip)
        held_x = which == "checkpoints" or at % 2 == 0
        X, x = (bx.pair(), x8) if held_x else (Strided(n, K, type_, pad, skip, x).t, x.double())
        Z, z = (bz.pair(), z8) if which == "checkpoints" or not held_x else (Strided(n, 2 * N, type_, pad, skip, z).t, z.double())
    dZ, dX, dW, H = out(n, 2 * N, type_, pad, skip), out(n, K, type_, pad, skip), out(K, 2 * N, type_, pad, skip), out(n, N, type_, pad, skip)
    db = torch.empty(2 * N, device="cuda")
    g.gcn_gated_backward(X, W.t, Z, dH.t, dZ.t, dX=dX.t, dW=dW.t, dbias=db, act=code(g, act), H=H.t)
    want = gated_back64(x, W.t.double().cpu(), z, dH.t.double().cpu(), act, type_)
    got = dict(dZ=dZ.t, dX=dX.t, dW=dW.t, H=H.t, dbias=db)
    u = UNIT[type_]
    for name, t in got.items():
        ref, off = want[name]
        check(t, ref, off + 1e-37 if name == "dbias" else off + u * (ref.abs() + off) + TINY[type_], name)
    for t in (dZ, dX, dW, H):
        assert t.outside_is_untouched()
    for one in ("dX", "dW", "dbias", "H"):                            # each by itself is the same
        alone = torch.empty_like(got[one])
        g.gcn_gated_backward(X if one == "dW" else None, W.t if one == "dX" else None, Z, dH.t, dZ.t if one in ("dX", "dW") else None, act=code(g, act),
                             **{one: alone})
        assert torch.equal(alone, got[one]), one


@pytest.mark.parametrize("type_", ALL)
@pytest.mark.parametrize("at", range(len(GATED)))
def test_backward_in_place(type_, at):
    """dZ in the place of Z, H in that of dH (dR in that of dY): the same bits, whatever lies beside a row's end in its rows."""
    g = lib()
    n, _, N, pad, skip = GATED[at]
    act = ACTS[at % 4]
    gen = gen_of("in place", type_, at)
    z, dh = normal(gen, (n, 2 * N), type_), normal(gen, (n, N), type_)
    Z, dH, dZ, H = Strided(n, 2 * N, type_, pad, skip, z), Strided(n, N, type_, pad, skip, dh), out(n, 2 * N, type_, pad, skip), out(n, N, type_, pad, skip)
    db, again = torch.empty(2, 2 * N, device="cuda")
    g.gcn_gated_backward(None, None, Z.t, dH.t, dZ.t, dbias=db, act=code(g, act), H=H.t)
    g.gcn_gated_backward(None, None, Z.t, dH.t, Z.t, dbias=again, act=code(g, act), H=dH.t)
    assert torch.equal(Z.t, dZ.t) and torch.equal(dH.t, H.t) and torch.equal(db, again)
    bz, _ = kept(z, type_, pad, skip)
    dY, dZ, dR = Strided(n, 2 * N, type_, pad, skip, normal(gen, (n, 2 * N), type_)), out(n, 2 * N, type_, pad, skip), out(n, 2 * N, type_, pad, skip)
    g.gcn_checkpoint_linear_backward(None, None, bz.pair(), dY.t, dZ.t, dbias=db, act=g.ACT_SILU, dR=dR.t, rho=0.5)
    g.gcn_checkpoint_linear_backward(None, None, bz.pair(), dY.t, dY.t, dbias=again, act=g.ACT_SILU)
    assert torch.equal(dY.t, dZ.t) and torch.equal(db, again)


@pytest.mark.parametrize("act", ACTS)
def test_gated_gradient_against_differences(act):
    """Along a random direction of all inputs, against the quotient of differences of the plain form in 64 bits (step 1e-6, so that no ReLU's corner lies
    between the two: the quotient is off by about 1e-9 of the terms' size)."""
    g = lib()
    n, K, N = 37, 50, 29
    gen = gen_of("gated differences", act)
    X, W, C = normal(gen, (n, K), "f32"), normal(gen, (K, 2 * N), "f32") * K ** -0.5, normal(gen, (n, N), "f32")
    b = normal(gen, (2 * N,), "f32")
    D = [torch.randn(t.shape, generator=gen, dtype=torch.float64) for t in (X, W, b)]
    forms = [t.double() for t in (X, W, b)]

    def z_at(h):
        x, w, c = (t + h * d for t, d in zip(forms, D))
        return x @ w + c

    def value(h):
        z = z_at(h)
        return float((C.double() * act64(z[:, :N], act) * z[:, N:]).sum())
    step = 1e-6
    if act == "relu":
        assert not bool(((z_at(step)[:, :N] > 0) != (z_at(-step)[:, :N] > 0)).any())
    quotient = (value(step) - value(-step)) / (2 * step)
    dev = [t.cuda() for t in (X, W, b)]
    H, Z, dZ = torch.empty(n, N, device="cuda"), torch.empty(n, 2 * N, device="cuda"), torch.empty(n, 2 * N, device="cuda")
    g.gcn_gated_forward(dev[0], dev[1], H, bias=dev[2], act=code(g, act), Z=Z)
    grads = [torch.empty_like(t) for t in dev]
    again = torch.empty_like(H)
    g.gcn_gated_backward(dev[0], dev[1], Z, C.cuda(), dZ, dX=grads[0], dW=grads[1], dbias=grads[2], act=code(g, act), H=again)
    terms = [(gr.double().cpu() * d) for gr, d in zip(grads, D)]
    got, size = sum(float(t.sum()) for t in terms), sum(float(t.abs().sum()) for t in terms)
    assert abs(got - quotient) <= 100 * EPS * size + 1e-7 * abs(quotient) + 1e-7
    assert bool(((again - H).abs() <= 4 * EPS * H.abs() + 1e-30).all())


@pytest.mark.parametrize("type_", ALL)
@pytest.mark.parametrize("n,K,N", [(5, 64, 48), (300, 200, 130), (4, 2048, 64), (1500, 128, 640)])
def test_gated_special_values_and_places(type_, n, K, N):
    """Infinities and NaN stay in their rows; dZ in the place of Z and H in the place of dH give the same bits."""
    g = lib()
    gen = gen_of("gated special", type_, n)
    X, W = normal(gen, (n, K), type_).cuda(), normal(gen, (K, 2 * N), type_, K ** -0.5).cuda()
    base, Z = torch.empty(n, N, dtype=TYPES[type_], device="cuda"), torch.empty(n, 2 * N, dtype=TYPES[type_], device="cuda")
    g.gcn_gated_forward(X, W, base, act=g.ACT_RELU, Z=Z)
    Y = X.clone()
    Y[1, 3], Y[2, K - 1] = float("nan"), float("inf")
    H, Zs = torch.empty_like(base), torch.empty_like(Z)
    g.gcn_gated_forward(Y, W, H, act=g.ACT_RELU, Z=Zs)
    keep = [i for i in range(n) if i not in (1, 2)]
    assert torch.equal(H[keep], base[keep]) and torch.equal(Zs[keep], Z[keep])
    assert bool(torch.isnan(Zs[1]).all()) and bool(torch.isnan(H[1]).all())
    there = W[K - 1] != 0
    assert torch.equal(Zs[2][there].float(), torch.where(W[K - 1][there] > 0, 1.0, -1.0) * float("inf"))
    dH = normal(gen, (n, N), type_).cuda()
    dZ, dX, dW, Hb = torch.empty_like(Z), torch.empty_like(X), torch.empty_like(W), torch.empty_like(base)
    g.gcn_gated_backward(X, W, Z, dH, dZ, dX=dX, dW=dW, H=Hb, act=g.ACT_GELU)
    z, dh, dx, dw = Z.clone(), dH.clone(), torch.empty_like(X), torch.empty_like(W)
    g.gcn_gated_backward(X, W, z, dh, z, dX=dx, dW=dw, H=dh, act=g.ACT_GELU)
    assert torch.equal(dx, dX) and torch.equal(dw, dW) and torch.equal(z, dZ) and torch.equal(dh, Hb)


# ---- linear layers' backward pass from checkpoints ------------------------------------------------------------------
@pytest.mark.parametrize("type_", ALL)
@pytest.mark.parametrize("at", range(len(GATED)))
def test_checkpoint_linear_backward(type_, at):
    """The bits that gcn_linear_backward gives of what the checkpoints stand for, but for the order of the sums of dW and dbias; and the formula's gradients."""
    g = lib()
    n, K, N, pad, skip = GATED[at]
    act = ACTS[(at + 2 + ALL.index(type_)) % 4]
    rho = 0.5
    gen = gen_of("checkpoint back", type_, at)
    bx, x = kept(normal(gen, (n, K), type_), type_, pad, skip)
    bz, z = kept(normal(gen, (n, N), type_), type_, pad, skip)
    W = Strided(K, N, type_, pad, skip, normal(gen, (K, N), type_, K ** -0.5))
    dY = Strided(n, N, type_, pad, skip, normal(gen, (n, N), type_))
    dZ, dX, dW, dR = out(n, N, type_, pad, skip), out(n, K, type_, pad, skip), out(K, N, type_, pad, skip), out(n, N, type_, pad, skip)
    db = torch.empty(N, device="cuda")
    g.gcn_checkpoint_linear_backward(bx.pair(), W.t, bz.pair(), dY.t, dZ.t, dX=dX.t, dW=dW.t, dbias=db, act=code(g, act), dR=dR.t, rho=rho)
    dt = TYPES[type_]
    like = {k: torch.empty_like(v) for k, v in dict(dX=dX.t, dW=dW.t, dbias=db, dR=dR.t).items()}
    dZ2 = torch.empty(n, N, dtype=dt, device="cuda")
    g.gcn_linear_backward(x.to(dt).cuda(), W.t, z.to(dt).cuda(), dY.t, dZ2, act=code(g, act), rho=rho, **like)
    assert torch.equal(like["dX"], dX.t) and torch.equal(like["dR"], dR.t)
    w, dy, u = W.t.double().cpu(), dY.t.double().cpu(), UNIT[type_]
    dz = dy * slope64(z, act)
    near = 8 * EPS * (z.abs() + 2) * dy.abs()
    # (the sums over the rows go in another order where rows are short)
    check(db, dz.sum(0), near.sum(0) * (act != "none") + (n + 2) * EPS * (dz.abs() + near).sum(0) + 1e-37, "dbias")
    dz_off = torch.zeros_like(dz) if act == "none" else near + u * (dz.abs() + near) + TINY[type_]
    size = dz.abs() + dz_off
    ref, off = x.t() @ dz, x.t().abs() @ dz_off + (n + 2) * EPS * (x.t().abs() @ size)
    check(dW.t, ref, off + u * (ref.abs() + off) + TINY[type_], "dW")
    ref, off = dz @ w.t(), dz_off @ w.t().abs() + (N + 2) * EPS * (size @ w.t().abs())
    check(dX.t, ref, off + u * (ref.abs() + off) + TINY[type_], "dX")
    for t in (dZ, dX, dW, dR):
        assert t.outside_is_untouched()
    # one of the two as elements
    got = torch.empty_like(dW.t)
    g.gcn_checkpoint_linear_backward(bx.pair(), W.t, z.to(dt).cuda(), dY.t, dZ2, dW=got, act=code(g, act))
    assert torch.equal(got, dW.t)
    g.gcn_checkpoint_linear_backward(x.to(dt).cuda(), W.t, bz.pair(), dY.t, dZ2, dW=got, act=code(g, act))
    assert torch.equal(got, like["dW"])


def test_checkpoint_that_stands_for_nan():
    """A group that was not finite makes its columns of dW NaN and no others; in Z its elements' rows of dX."""
    g = lib()
    gen = gen_of("nan groups")
    n, K, N = 200, 192, 128
    x = normal(gen, (n, K), "bf16")
    x[17, 70] = float("inf")
    z = normal(gen, (n, N), "bf16")
    z[5, 127] = float("nan")
    bx, bz = Bytes(n, K), Bytes(n, N)
    g.gcn_checkpoint_pack(x.cuda(), *bx.pair())
    g.gcn_checkpoint_pack(z.cuda(), *bz.pair())
    W, dY = normal(gen, (K, N), "bf16").cuda(), normal(gen, (n, N), "bf16").cuda()
    e = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")
    dZ, dX, dW = e(n, N), e(n, K), e(K, N)
    g.gcn_checkpoint_linear_backward(bx.pair(), W, None, dY, None, dX=dX, dW=dW)
    bad = torch.isnan(dW).all(1).cpu()
    assert torch.equal(bad, (torch.arange(K) >= 64) & (torch.arange(K) < 128)) and bool(torch.isfinite(dW[~bad.cuda()]).all())
    g.gcn_checkpoint_linear_backward(None, W, bz.pair(), dY, dZ, dX=dX, act=g.ACT_SILU)
    assert bool(torch.isnan(dX[5]).all()) and bool(torch.isfinite(dX[torch.arange(n) != 5]).all())
    assert torch.equal(torch.isnan(dZ[5]).cpu(), torch.arange(N) >= 64)


# ---- products with weights in 4 bits --------------------------------------------------------------------------------
LINEAR4 = [(1, 1, 1, 32, 0, 0), (1, 64, 64, 64, 0, 0), (1, 1000, 300, 128, 0, 0), (1, 4096, 48, 32, 8, 0), (2, 4096, 40, 128, 8, 0), (3, 5, 7, 32, 0, 1), (16, 512, 1024, 64, 0, 0), (17, 33, 65, 32, 3, 0),
           (32, 160, 96, 64, 0, 8), (33, 160, 96, 128, 0, 8), (64, 64, 64, 32, 0, 0), (65, 128, 129, 64, 0, 0), (130, 602, 41, 128, 0, 0), (257, 96, 304, 32, 16, 0), (1000, 37, 8, 64, 0, 0),
           (2049, 72, 808, 32, 0, 0), (2049, 71, 801, 64, 1, 1), (1027, 520, 2048, 128, 0, 0), (20001, 48, 24, 64, 0, 0), (9, 3000, 17, 32, 0, 0), (8, 24, 20000, 64, 0, 0),
           (5, 20000, 24, 128, 0, 0), (40, 8200, 72, 64, 0, 0), (100, 3, 50, 32, 0, 0), (70, 7, 200, 128, 0, 1), (301, 1, 9, 64, 2, 0), (20000, 3, 300, 32, 0, 0), (70001, 2, 5, 64, 0, 0)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("type_", ALL)
@pytest.mark.parametrize("at", range(len(LINEAR4)))
def test_linear4_forward(type_, at, gated):
    g = lib()
    n, K, N, group, pad, skip = LINEAR4[at]
    cols = 2 * N if gated else N
    act = ACTS[(at + ALL.index(type_)) % 4]
    rho = 1.0 if at % 4 < 2 else -0.75
    gen = gen_of("linear4", type_, at, gated)
    X = Strided(n, K, type_, pad, skip, normal(gen, (n, K), type_))
    Q, S, w = weights(normal(gen, (K, cols), type_, K ** -0.5), group, type_, pad, skip)
    b = normal(gen, (cols,), "f32").cuda() if at % 3 else None
    R = Strided(n, N, type_, pad, skip, normal(gen, (n, N), type_)) if at % 2 else None
    Y = out(n, N, type_, pad, skip)
    args = dict(group=group, bias=b, act=code(g, act), R=None if R is None else R.t, rho=rho, gated=gated)
    g.gcn_linear4_forward(X.t, Q, S, Y.t, **args)
    z, off = product_off(X.t.double().cpu(), w, None if b is None else b.double().cpu())
    if gated:
        y, y_off = gate64(z, off, act)
    else:
        y, y_off = act64(z, act), SLOPE_MOST * off + 8 * EPS * (z.abs() + 1e-30)
    if R is not None:
        r = rho * R.t.double().cpu()
        y, y_off = y + r, y_off + 2 * EPS * (r.abs() + y.abs())
    check(Y.t, y, y_off + UNIT[type_] * (y.abs() + y_off) + TINY[type_], "Y")
    assert Y.outside_is_untouched()
    again = out(n, N, type_, pad, skip)
    g.gcn_linear4_forward(X.t, Q, S, again.t, **args)
    assert torch.equal(again.t, Y.t), "the same call gives other bits"
    if R is not None:
        g.gcn_linear4_forward(X.t, Q, S, R.t, **args)
        assert torch.equal(R.t, Y.t) and R.outside_is_untouched()


@pytest.mark.parametrize("type_", ALL)
@pytest.mark.parametrize("n,K,N", [(3, 300, 72), (90, 300, 72)])
def test_linear4_special_values(type_, n, K, N):
    """Infinities and NaN of X stay in their rows, a scale that is NaN in its column; codes behind the last weight are not seen."""
    g = lib()
    gen = gen_of("linear4 special", type_, n)
    x = normal(gen, (n, K), type_)
    Q, S, w = weights(normal(gen, (K, N), type_), 64, type_, 0, 0)
    base, Y = (torch.empty(n, N, dtype=TYPES[type_], device="cuda") for _ in range(2))
    g.gcn_linear4_forward(x.cuda(), Q, S, base)
    assert K % 8 == 4
    dirty = Q.clone()
    dirty[-1] |= torch.tensor(0x77770000, dtype=torch.int32, device="cuda")
    g.gcn_linear4_forward(x.cuda(), dirty, S, Y)
    assert torch.equal(Y, base)
    x[1, 3], x[2, K - 1] = float("nan"), float("inf")
    g.gcn_linear4_forward(x.cuda(), Q, S, Y)
    keep = [i for i in range(n) if i not in (1, 2)]
    assert torch.equal(Y[keep], base[keep]) and bool(torch.isnan(Y[1]).all())
    last = w[K - 1].cuda()
    want = torch.where(last == 0, float("nan"), last.sign() * float("inf"))
    assert torch.equal(torch.nan_to_num(Y[2].double(), nan=7.0), torch.nan_to_num(want, nan=7.0))
    S = S.clone()
    S[1, 5] = float("nan")
    g.gcn_linear4_forward(x.cuda(), Q, S, Y)
    assert bool(torch.isnan(Y[:, 5]).all())
    others = [c for c in range(N) if c != 5]
    assert torch.equal(Y[keep][:, others], base[keep][:, others])


def test_linear4_fp32_large_and_small_rows():
    """fp32 rows of all magnitudes, next to the largest number and far below 1, keep 24 bits."""
    g = lib()
    gen = gen_of("linear4 sizes")
    for n in (7, 70):
        x = normal(gen, (n, 200), "f32") * torch.exp2(torch.linspace(-90, 110, n)).float()[:, None]
        x[0, 0], x[-1, :] = 1.0, 0
        x[-1, 3] = torch.finfo(torch.float32).max
        Q, S, w = weights(normal(gen, (200, 40), "f32", 0.01), 32, "f32", 0, 0)
        Y = torch.empty(n, 40, device="cuda")
        g.gcn_linear4_forward(x.cuda(), Q, S, Y, group=32)
        z, off = product_off(x.double(), w, None)
        check(Y, z, off + EPS * z.abs(), "Y")


def test_column_blocks_of_held_matrices():
    """A block of columns of weights in 4 bits is those columns of W: two gated halves that lie apart from one another are a layer each."""
    g = lib()
    gen = gen_of("blocks")
    n, K, N = 5, 256, 96
    X = normal(gen, (n, K), "bf16").cuda()
    Q, S, w = weights(normal(gen, (K, 2 * N), "bf16"), 64, "bf16", 0, 0)
    both, one, two = (torch.empty(n, c, dtype=torch.bfloat16, device="cuda") for c in (2 * N, N, N))
    g.gcn_linear4_forward(X, Q, S, both)
    g.gcn_linear4_forward(X, Q[:, :N], S[:, :N], one)
    g.gcn_linear4_forward(X, Q[:, N:], S[:, N:], two)
    assert torch.equal(both, torch.cat([one, two], 1))


# ---- together -------------------------------------------------------------------------------------------------------
class Block:
    """A student's block: X' = X + H W2 with H the gated block of X; trained from checkpoints, answering from 4-bit weights."""

    def __init__(self, n, f, m, type_, seed):
        gen = gen_of("block", type_, seed)
        self.n, self.f, self.m = n, f, m
        self.dt = TYPES[type_]
        self.W, self.W2 = normal(gen, (f, 2 * m), type_, f ** -0.5).cuda(), normal(gen, (m, f), type_, m ** -0.5).cuda()
        self.b = normal(gen, (2 * m,), "f32", 0.1).cuda()
        e = lambda *s, dt=self.dt: torch.zeros(*s, dtype=dt, device="cuda")
        self.X, self.dY = normal(gen, (n, f), type_).cuda(), normal(gen, (n, f), type_).cuda()
        self.Z, self.H, self.Y, self.dH, self.dZ, self.dX = e(n, 2 * m), e(n, m), e(n, f), e(n, m), e(n, 2 * m), e(n, f)
        self.dW, self.dW2, self.db = e(f, 2 * m), e(m, f), e(2 * m, dt=torch.float32)
        self.x8, self.z8 = Bytes(n, f).pair(), Bytes(n, 2 * m).pair()
        self.q, self.s = e(-(-f // 8), 2 * m, dt=torch.int32), e(-(-f // 64), 2 * m, dt=torch.bfloat16)
        self.q2, self.s2 = e(-(-m // 8), f, dt=torch.int32), e(-(-m // 64), f, dt=torch.bfloat16)
        self.H4, self.Y4 = e(n, m), e(n, f)
        self.outs = (self.Y, self.dX, self.dW, self.dW2, self.db, self.Y4, self.q, self.s, self.x8[0], self.z8[0])

    def step(self):
        g = lib()
        g.gcn_checkpoint_pack(self.X, *self.x8)
        g.gcn_gated_forward(self.X, self.W, self.H, bias=self.b, Z=self.Z)
        g.gcn_checkpoint_pack(self.Z, *self.z8)
        g.gcn_linear_forward(self.H, self.W2, self.Y, R=self.X)
        g.gcn_linear_backward(None, self.W2, None, self.dY, dX=self.dH)
        g.gcn_gated_backward(self.x8, self.W, self.z8, self.dH, self.dZ, dX=self.dX, dW=self.dW, dbias=self.db, H=self.H)
        g.gcn_linear_backward(self.H, None, None, self.dY, dW=self.dW2)
        g.gcn_linear4_pack(self.W, self.q, self.s)
        g.gcn_linear4_pack(self.W2, self.q2, self.s2)
        g.gcn_linear4_forward(self.X, self.q, self.s, self.H4, bias=self.b, act=g.ACT_SILU, gated=True)
        g.gcn_linear4_forward(self.H4, self.q2, self.s2, self.Y4, R=self.X)


@pytest.mark.parametrize("type_", ALL)
@pytest.mark.parametrize("n,f,m", [(7, 128, 200), (700, 128, 320)])
def test_a_block_trained_and_answering(type_, n, f, m):
    """The block's outputs and gradients against autograd in 64 bits, up to what 8 and 4 bits leave: the checkpoint is off by 1/254 of a group's largest number at most, about a
    hundredth of the elements' size; 4 bits by a tenth."""
    B = Block(n, f, m, type_, 0)
    B.step()
    X, W, W2, b = (t.double().cpu().requires_grad_() for t in (B.X, B.W, B.W2, B.b))
    z = X @ W + b
    h = act64(z[:, :m], "silu") * z[:, m:]
    y = h @ W2 + X
    rel = lambda a, r: float((a.double().cpu() - r).norm() / r.norm())
    dX, dW, dW2, db = torch.autograd.grad((h @ W2), (X, W, W2, b), B.dY.double().cpu())
    assert rel(B.Y, y.detach()) < 0.01
    for got, want in ((B.dX, dX), (B.dW, dW), (B.dW2, dW2), (B.db, db)):
        assert rel(got, want) < 0.05
    assert rel(B.Y4, y.detach()) < 0.25


@pytest.mark.parametrize("type_", ALL)
def test_a_block_on_streams_and_in_graphs(type_):
    """On a stream of the caller's and captured and replayed with new inputs, two graphs in turn, with eager work between: the eager results bit by bit."""
    blocks = [Block(300, 128, 200, type_, 1), Block(9, 256, 136, type_, 2)]
    side = torch.cuda.Stream()
    for B in blocks:
        B.step()
    torch.cuda.synchronize()
    graphs = []
    for B in blocks:
        first = [o.clone() for o in B.outs]
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for o in B.outs:
                o.zero_()
            B.step()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, B.outs))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            B.step()
        graphs.append(graph)
    gen = gen_of("graphs", type_)
    for round_ in range(3):
        for B, graph in zip(blocks, graphs):
            B.X.copy_(normal(gen, tuple(B.X.shape), type_))
            B.W.mul_(0.9)
            B.step()
            torch.cuda.synchronize()
            want = [o.clone() for o in B.outs]
            for o in B.outs:
                o.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, B.outs)), round_


def test_offsets_beyond_32_bits():
    """Rows, codes, scales and words that lie more than 2^32 bytes behind the first."""
    g = lib()
    gen = gen_of("far held")
    n, K, N = 3, 72, 40
    ld = (1 << 30) + 8
    buf = torch.empty(3 * ld, dtype=torch.bfloat16, device="cuda")
    far = buf.as_strided((n, K), (ld, 1))
    x = normal(gen, (n, K), "bf16").cuda()
    far.copy_(x)
    W = normal(gen, (K, 2 * N), "bf16").cuda()
    H, want = (torch.empty(n, N, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    g.gcn_gated_forward(far, W, H)
    g.gcn_gated_forward(x, W, want)
    assert torch.equal(H, want)
    near = Bytes(n, K)
    g.gcn_checkpoint_pack(x, *near.pair())
    ld8 = (1 << 31) + 64
    codes = buf.view(torch.int8)[:2 * ld8 + K + 8].as_strided((n, K), (ld8, 1))
    scales = buf[4096:].as_strided((n, 2), (ld - 5, 1))
    assert codes.dtype == torch.int8
    g.gcn_checkpoint_pack(x, codes, scales)
    assert torch.equal(codes, near.codes) and torch.equal(scales, near.scales)
    back, dY = torch.empty_like(x), normal(gen, (n, N), "bf16").cuda()
    g.gcn_checkpoint_unpack(codes, scales, back)
    assert torch.equal(back.double().cpu(), near.values(torch.bfloat16))
    dW, dW2 = (torch.empty(K, N, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    g.gcn_checkpoint_linear_backward((codes, scales), None, None, dY, dW=dW)
    g.gcn_checkpoint_linear_backward(near.pair(), None, None, dY, dW=dW2)
    assert torch.equal(dW, dW2)
    del codes, scales, far
    words = buf.view(torch.int32)
    Q, S, w = weights(normal(gen, (24, N), "bf16"), 32, "bf16", 0, 0)
    ldq = (1 << 29) + 16
    Qf = words.as_strided((3, N), (ldq, 1))
    Qf.copy_(Q)
    Y, want = (torch.empty(n, N, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for rows in (n, 70):
        xs = normal(gen, (rows, 24), "bf16").cuda()
        Y, want = (torch.empty(rows, N, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        g.gcn_linear4_forward(xs, Qf, S, Y, group=32)
        g.gcn_linear4_forward(xs, Q, S, want, group=32)
        assert torch.equal(Y, want)
