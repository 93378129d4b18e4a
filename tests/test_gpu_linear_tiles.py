"""Every tile of the linear layers' products, in each of the three directions, with and without a split sum, through registers and from memory to LDS, and the
kernels for few rows at every width of their strips, against products in 64 bits.  That the sizes take the tiles that they stand for is tested without a GPU.

Tolerances are derived as in test_gpu_operators.py."""
import pytest

torch = pytest.importorskip("torch")

from linear_tiles import PRODUCTS
from test_gpu_operators import EPS, SLOPE_MOST, TINY, UNIT, Strided, act64, check, code, gen_of, lib, normal, out, slope64

pytestmark = pytest.mark.gpu

CASES = [(t, p) for p in PRODUCTS for t in (["bf16", "f16"] if p[0] == "16" else ["f32"])]
NAMES = [f"{t}-{p[2]}-{'whole' if p[1] else 'ragged'}-{p[3]}" for t, p in CASES]


def matrix(rows, cols, type_, whole, value=None):
    """Rows at 16-byte addresses, or at odd ones."""
    pad, skip = (-cols % 8, 0) if whole else (0, 1)
    return out(rows, cols, type_, pad, skip) if value is None else Strided(rows, cols, type_, pad, skip, value)


def forward(type_, whole, n, K, N, act):
    g = lib()
    gen = gen_of("tiles", type_, n, K, N)
    X, W = matrix(n, K, type_, whole, normal(gen, (n, K), type_)), matrix(K, N, type_, whole, normal(gen, (K, N), type_, K ** -0.5))
    R, b = matrix(n, N, type_, whole, normal(gen, (n, N), type_)), normal(gen, (N,), "f32").cuda()
    Y, Z = matrix(n, N, type_, whole), matrix(n, N, type_, whole)
    g.gcn_linear_forward(X.t, W.t, Y.t, bias=b, act=code(g, act), R=R.t, rho=-0.75, Z=Z.t)
    x, w = X.t.double(), W.t.double()
    z, size = (x @ w + b.double()).cpu(), (x.abs() @ w.abs() + b.double().abs()).cpu()
    off, r = (K + 2) * EPS * size, -0.75 * R.t.double().cpu()
    u = UNIT[type_]
    check(Z.t, z, off + u * (z.abs() + off) + TINY[type_], "Z")
    y = act64(z, act) + r
    inner = SLOPE_MOST * off + 8 * EPS * (z.abs() + 1e-30) + 2 * EPS * r.abs()
    check(Y.t, y, inner + u * (y.abs() + inner) + TINY[type_], "Y")
    assert Y.outside_is_untouched() and Z.outside_is_untouched()
    again = matrix(n, N, type_, whole)
    g.gcn_linear_forward(X.t, W.t, again.t, bias=b, act=code(g, act), R=R.t, rho=-0.75)
    assert torch.equal(again.t, Y.t), "the same call gives other bits"


@pytest.mark.parametrize("type_,product", CASES, ids=NAMES)
def test_forward(type_, product):
    _, whole, _, _, M, N, K = product
    forward(type_, whole, M, K, N, "gelu")


@pytest.mark.parametrize("which", ["dX", "dW"])
@pytest.mark.parametrize("type_,product", CASES, ids=NAMES)
def test_backward(type_, product, which):
    g = lib()
    _, whole, _, _, M, N, K = product
    n, f_in, f_out = (M, N, K) if which == "dX" else (K, M, N)
    gen = gen_of("tilesback", which, type_, M, N, K)
    Z, dY = (matrix(n, f_out, type_, whole, normal(gen, (n, f_out), type_)) for _ in range(2))
    shape = (f_in, f_out) if which == "dX" else (n, f_in)
    other = matrix(*shape, type_, whole, normal(gen, shape, type_, f_out ** -0.5 if which == "dX" else 1.0))
    dZ = matrix(n, f_out, type_, whole)
    d = matrix(n, f_in, type_, whole) if which == "dX" else matrix(f_in, f_out, type_, whole)

    def call(to):
        if which == "dX":
            g.gcn_linear_backward(None, other.t, Z.t, dY.t, dZ.t, dX=to, act=g.ACT_SILU)
        else:
            g.gcn_linear_backward(other.t, None, Z.t, dY.t, dZ.t, dW=to, act=g.ACT_SILU)
    call(d.t)
    z, dy, o = Z.t.double(), dY.t.double(), other.t.double()
    dz = dy * slope64(z, "silu")
    near = 8 * EPS * (z.abs() + 2) * dy.abs()
    dz_off = near + UNIT[type_] * (dz.abs() + near) + TINY[type_]
    # dZ's own error goes through the product, and the product is a sum of K terms
    each = dz_off + (K + 2) * EPS * (dz.abs() + dz_off)
    ref, off = (dz @ o.t(), each @ o.t().abs()) if which == "dX" else (o.t() @ dz, o.t().abs() @ each)
    check(d.t, ref.cpu(), (off + UNIT[type_] * (ref.abs() + off) + TINY[type_]).cpu(), which)
    assert d.outside_is_untouched() and dZ.outside_is_untouched()
    again = torch.empty_like(d.t)
    call(again)
    assert torch.equal(again, d.t), "the same call gives other bits"


# 16, 32 and 64 columns a strip for up to 16 and 32 rows: the widest that give each of 256 compute units one, and a last strip that a row's end cuts
@pytest.mark.parametrize("type_", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("n,K,N", [(1, 300, 4100), (16, 1031, 8209), (31, 517, 8200), (13, 700, 16400), (32, 1029, 16421), (17, 64, 20000)])
def test_few_rows(type_, whole, n, K, N):
    forward(type_, whole, n, K, N, "silu")


@pytest.mark.parametrize("type_", ["f32", "bf16"])
def test_tiles_of_rows_far_apart(type_):
    """Rows of every operand more than 2^32 elements behind the first: the tiles' products in each direction."""
    g = lib()
    n, K, N = 40, 24, 48
    ld = (1 << 27) + 8 if type_ == "bf16" else (1 << 27) + 4
    gen = gen_of("farther", type_)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[type_]

    def far(cols, value=None):
        t = torch.empty((n - 1) * ld + cols, dtype=dt, device="cuda").as_strided((n, cols), (ld, 1))
        return t if value is None else t.copy_(value)
    x, dy, w = normal(gen, (n, K), type_).cuda(), normal(gen, (n, N), type_).cuda(), normal(gen, (K, N), type_).cuda()
    e = lambda *s: torch.empty(*s, dtype=dt, device="cuda")
    y0, z0, dz0, dx0, dw0 = e(n, N), e(n, N), e(n, N), e(n, K), e(K, N)
    g.gcn_linear_forward(x, w, y0, act=g.ACT_SILU, Z=z0)
    g.gcn_linear_backward(x, w, z0, dy, dz0, dX=dx0, dW=dw0, act=g.ACT_SILU)
    X, Y = far(K, x), far(N)
    g.gcn_linear_forward(X, w, Y, act=g.ACT_SILU)
    assert torch.equal(Y, y0)
    Y.copy_(dy)
    dX, dw = far(K), e(K, N)
    g.gcn_linear_backward(X, w, z0, Y, Y, dX=dX, dW=dw, act=g.ACT_SILU)      # dY's place takes dZ
    assert torch.equal(dX, dx0) and torch.equal(dw, dw0) and torch.equal(Y, dz0)
