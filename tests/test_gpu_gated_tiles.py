"""Every kernel of the gated blocks and of the products with weights in 4 bits, at sizes that gated_tiles.py lists, against products in 64 bits.

Tolerances are derived as in test_gpu_operators.py."""
import pytest

torch = pytest.importorskip("torch")

import held
from gated_tiles import FEW4, GATED, TILES4
from linear_tiles import PRODUCTS
from test_gpu_gated import gate64, kept
from test_gpu_linear_tiles import matrix
from test_gpu_operators import EPS, SLOPE_MOST, TINY, UNIT, act64, check, code, gen_of, lib, normal

pytestmark = pytest.mark.gpu


def by_types(sizes):
    return [(t, p) for p in sizes for t in (["bf16", "f16"] if p[0] == "16" else ["f32"])]


def names(cases):
    return ["-".join(str(x) for x in (t, *p[1:])) for t, p in cases]


def sums(x, w, b):
    """x w + b in 64 bits, on the GPU, and how far its sum in 32 may be off; both on the CPU."""
    z, size = x @ w + b, x.abs() @ w.abs() + b.abs()
    return z.cpu(), ((x.shape[1] + 2) * EPS * size).cpu()


@pytest.mark.parametrize("type_,p", by_types(GATED), ids=names(by_types(GATED)))
def test_gated_tiles(type_, p):
    g = lib()
    _, whole, _, _, n, N, K = p
    gen = gen_of("gated tiles", type_, n, N, K)
    X, W = matrix(n, K, type_, whole, normal(gen, (n, K), type_)), matrix(K, 2 * N, type_, whole, normal(gen, (K, 2 * N), type_, K ** -0.5))
    b = normal(gen, (2 * N,), "f32").cuda()
    H, Z = matrix(n, N, type_, whole), matrix(n, 2 * N, type_, whole)
    g.gcn_gated_forward(X.t, W.t, H.t, bias=b, act=g.ACT_GELU, Z=Z.t)
    z, off = sums(X.t.double(), W.t.double(), b.double())
    h, h_off = gate64(z, off, "gelu")
    u = UNIT[type_]
    check(Z.t, z, off + u * (z.abs() + off) + TINY[type_], "Z")
    check(H.t, h, h_off + u * (h.abs() + h_off) + TINY[type_], "H")
    assert H.outside_is_untouched() and Z.outside_is_untouched()
    again = matrix(n, N, type_, whole)
    g.gcn_gated_forward(X.t, W.t, again.t, bias=b, act=g.ACT_GELU)
    assert torch.equal(again.t, H.t), "the same call gives other bits"


# both halves in pieces of 128 bytes and narrower ones, shared and not; n, f_out, f_in
@pytest.mark.parametrize("type_", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("n,N,K", [(1, 4100, 2100), (16, 2051, 4099), (5, 16500, 300), (31, 2049, 2065), (32, 8200, 130), (17, 1030, 520), (3, 4097, 1030), (9, 101, 8200)])
def test_gated_few_rows(type_, whole, n, N, K):
    test_gated_tiles(type_, (None, whole, None, None, n, N, K))


def four_bits(g, gen, K, cols, group, type_):
    """Weights in 4 bits laid out by the library, and what they stand for, in 64 bits on the GPU."""
    W = normal(gen, (K, cols), type_, K ** -0.5).cuda()
    Q, S = torch.empty(-(-K // 8), cols, dtype=torch.int32, device="cuda"), torch.empty(-(-K // group), cols, dtype=torch.bfloat16, device="cuda")
    g.gcn_linear4_pack(W, Q, S, group=group)
    q = (Q[:, None, :] >> torch.arange(0, 32, 4, dtype=torch.int32, device="cuda")[None, :, None]) & 15
    q = q.reshape(-1, cols)[:K].long()
    v = held.LEVELS.cuda()[q & 7]
    return Q, S, torch.where(q >= 8, -v, v) * S.double().repeat_interleave(group, 0)[:K]


def product4(type_, n, cols, K, group, gated, act="silu"):
    g = lib()
    gen = gen_of("4 bits", type_, n, cols, K, group, gated)
    N = cols // 2 if gated else cols
    X = matrix(n, K, type_, False, normal(gen, (n, K), type_))
    Q, S, w = four_bits(g, gen, K, cols, group, type_)
    b, R = normal(gen, (cols,), "f32").cuda(), matrix(n, N, type_, False, normal(gen, (n, N), type_))
    Y = matrix(n, N, type_, False)
    args = dict(group=group, bias=b, act=code(g, act), R=R.t, rho=-0.75, gated=gated)
    g.gcn_linear4_forward(X.t, Q, S, Y.t, **args)
    z, off = sums(X.t.double(), w, b.double())
    y, y_off = gate64(z, off, act) if gated else (act64(z, act), SLOPE_MOST * off + 8 * EPS * (z.abs() + 1e-30))
    r = -0.75 * R.t.double().cpu()
    y, y_off = y + r, y_off + 2 * EPS * (r.abs() + y.abs())
    check(Y.t, y, y_off + UNIT[type_] * (y.abs() + y_off) + TINY[type_], "Y")
    assert Y.outside_is_untouched()
    again = torch.empty_like(Y.t)
    g.gcn_linear4_forward(X.t, Q, S, again, **args)
    assert torch.equal(again, Y.t), "the same call gives other bits"


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("type_,p", by_types(FEW4), ids=names(by_types(FEW4)))
def test_few_rows_of_4_bits(type_, p, gated):
    _, _, _, _, n, cols, K = p
    product4(type_, n, cols, K, (32, 64, 128)[(K + gated) % 3], gated)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("type_,p", by_types(TILES4), ids=names(by_types(TILES4)))
def test_tiles_of_4_bits(type_, p, group, gated):
    _, _, n, cols, K = p
    product4(type_, n, cols, K, group, gated, "gelu")


HELD = [(t, p) for t, p in [("f32", p) for p in PRODUCTS if p[0] == "f32"] + [("bf16", p) for p in PRODUCTS if p[0] == "16" and p[3] == 1]]


@pytest.mark.parametrize("type_,p", HELD, ids=names(HELD))
def test_weights_gradient_from_a_checkpoint(type_, p):
    """dW = X^T dY of every tile, X a checkpoint of as many columns as the list says and of the next multiple of four (which fp32 products take from the codes)."""
    g = lib()
    _, whole, _, _, M, N, K = p
    for f_in in (M, -(-M // 4) * 4):
        gen = gen_of("held dW", type_, f_in, N, K)
        bx, x = kept(normal(gen, (K, f_in), type_), type_, 0 if whole else 3, 0 if whole else 1)
        dY = matrix(K, N, type_, whole, normal(gen, (K, N), type_))
        dW = matrix(f_in, N, type_, whole)
        g.gcn_checkpoint_linear_backward(bx.pair(), None, None, dY.t, dW=dW.t)
        x, dy = x.cuda(), dY.t.double()
        ref, off = x.t() @ dy, (K + 2) * EPS * (x.abs().t() @ dy.abs())
        check(dW.t, ref.cpu(), (off + UNIT[type_] * (ref.abs() + off) + TINY[type_]).cpu(), "dW")
        assert dW.outside_is_untouched()
        again = torch.empty_like(dW.t)
        g.gcn_checkpoint_linear_backward(bx.pair(), None, None, dY.t, dW=again)
        assert torch.equal(again, dW.t), "the same call gives other bits"


PADDED = [("bf16", p) for p in PRODUCTS if p[0] == "16" and p[1]]


@pytest.mark.parametrize("type_,p", PADDED, ids=names(PADDED))
def test_weights_gradient_of_padded_rows(type_, p):
    """dW of X a checkpoint of f_in columns that do not fill 16 bytes: its restored rows do, and what lies behind them, here NaN of a call before, is no part of a result."""
    g = lib()
    _, _, _, _, M, N, K = p
    gen = gen_of("padded dW", type_, M, N, K)
    dY = matrix(K, N, type_, True, normal(gen, (K, N), type_))
    codes = torch.ones(K, M, dtype=torch.int8, device="cuda")
    scales = torch.full((K, -(-M // g.CHECKPOINT_GROUP)), float("nan"), dtype=torch.bfloat16, device="cuda")
    lost = torch.empty(M, N, dtype=dY.t.dtype, device="cuda")
    g.gcn_checkpoint_linear_backward((codes, scales), None, None, dY.t, dW=lost)
    assert torch.isnan(lost).all()
    for f_in in (M - 1, M - 7):
        bx, x = kept(normal(gen, (K, f_in), type_), type_, 3, 1)
        dW = matrix(f_in, N, type_, False)
        g.gcn_checkpoint_linear_backward(bx.pair(), None, None, dY.t, dW=dW.t)
        x, dy = x.cuda(), dY.t.double()
        ref, off = x.t() @ dy, (K + 2) * EPS * (x.abs().t() @ dy.abs())
        check(dW.t, ref.cpu(), (off + UNIT[type_] * (ref.abs() + off) + TINY[type_]).cpu(), "dW")
        assert dW.outside_is_untouched()
