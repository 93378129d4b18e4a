"""Gated blocks and products with weights in 4 bits on numbers whose sums are exact in 32 bits, whatever their order: results are equal to those in 64 bits, so that a value of k left out, taken twice or
cut short shows at any length.  And backward passes against the products of the dZ that they leave."""
import pytest

torch = pytest.importorskip("torch")

import held
from gated_tiles import FEW4, GATED, TILES4
from test_gpu_gated import kept
from test_gpu_gated_tiles import by_types, names
from test_gpu_linear_tiles import matrix
from test_gpu_operators import EPS, TINY, TYPES, UNIT, check, gen_of, lib, normal, out

pytestmark = pytest.mark.gpu


def on_gpu(*key):
    return torch.Generator(device="cuda").manual_seed(gen_of(*key).initial_seed())


def whole(gen, shape):
    """Whole numbers up to 3."""
    return torch.randint(-3, 4, shape, generator=gen, device="cuda").double()


def one_of_a_row(gen, n, k):
    """Rows with a single number, of 24 bits: in turn at the end of k, about a border of 128 values of it, and anywhere."""
    i = torch.arange(n, device="cuda")
    borders = (128 * ((i * 7) % (k // 128 + 1)) - i // 3 % 2).clamp(0, k - 1)
    at = torch.where(i % 3 == 0, (k - 1 - i // 3 % 64).clamp(min=0), torch.where(i % 3 == 1, borders, torch.randint(k, (n,), generator=gen, device="cuda")))
    x = torch.zeros(n, k, dtype=torch.float64, device="cuda")
    bits = torch.randint(1 << 23, 1 << 24, (n,), generator=gen, device="cuda").double() * 2.0 ** -23
    x[i, at] = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.5, -bits, bits)
    return x


def gated_results(z, N, type_):
    """What the block's H is: the product of two sums of 32 bits, rounded to it, and then to the type."""
    z = z.float()
    return (z[:, :N] * z[:, N:]).to(TYPES[type_])


def gated_is_exact(type_, rows, n, N, K, x, w):
    g = lib()
    X, W = matrix(n, K, type_, rows, x), matrix(K, 2 * N, type_, rows, w)
    H, Z = matrix(n, N, type_, rows), matrix(n, 2 * N, type_, rows)
    g.gcn_gated_forward(X.t, W.t, H.t, act=g.ACT_NONE, Z=Z.t)
    z = x @ w
    assert torch.equal(Z.t, z.to(TYPES[type_])) and torch.equal(H.t, gated_results(z, N, type_))


@pytest.mark.parametrize("type_,p", by_types(GATED), ids=names(by_types(GATED)))
def test_gated_tiles(type_, p):
    _, rows, _, _, n, N, K = p
    gen = on_gpu("exact", type_, n, N, K)
    signs = 2 * torch.randint(0, 2, (K, 2 * N), generator=gen, device="cuda") - 1
    gated_is_exact(type_, rows, n, N, K, whole(gen, (n, K)), (torch.randint(1, 3, (K, 2 * N), generator=gen, device="cuda") * signs).double())
    if type_ == "f32":                                                # all bits of what is split in three
        gated_is_exact(type_, rows, n, N, K, one_of_a_row(gen, n, K), signs * torch.exp2(torch.randint(-3, 4, (K, 2 * N), generator=gen, device="cuda").double()))


def weights(gen, K, cols, group, places):
    """Q and S of random codes among `places`, with scales of 1/2, 1 and 2, and what they stand for."""
    code = torch.tensor(places, device="cuda")[torch.randint(len(places), (K, cols), generator=gen, device="cuda")] + 8 * torch.randint(0, 2, (K, cols), generator=gen, device="cuda")
    S = torch.exp2(torch.randint(-1, 2, (-(-K // group), cols), generator=gen, device="cuda").float()).bfloat16()
    padded = torch.nn.functional.pad(code, (0, 0, 0, -K % 8)).view(-1, 8, cols)
    Q = (padded << torch.arange(0, 32, 4, device="cuda")[None, :, None]).sum(1)
    v = held.LEVELS.cuda()[code & 7]
    return torch.where(Q >= 1 << 31, Q - (1 << 32), Q).int(), S, torch.where(code >= 8, -v, v) * S.double().repeat_interleave(group, 0)[:K]


def four_bits_are_exact(type_, n, cols, K, group, gated, x, gen, places, R=None):
    """`cols` of the weights, as wide as they are; x whole numbers times places of halves times scales of 1/2 and more: multiples of 1/4 far below 2^22."""
    g = lib()
    N = cols // 2 if gated else cols
    Q, S, w = weights(gen, K, cols, group, places)
    X, Y = matrix(n, K, type_, False, x), matrix(n, N, type_, False)
    g.gcn_linear4_forward(X.t, Q, S, Y.t, group=group, gated=gated, R=R, rho=2.0)
    z = x @ w
    if R is not None:
        z = z + 2 * R.double()
    assert torch.equal(Y.t, gated_results(z, N, type_) if gated else z.to(TYPES[type_]))
    assert Y.outside_is_untouched()


FOUR = [(t, p[-3:], group) for (t, p) in by_types(FEW4) for group in ((32, 64, 128)[p[-1] % 3],)] + [(t, p[-3:], group) for (t, p) in by_types(TILES4) for group in (32, 64, 128)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("type_,p,group", FOUR, ids=["-".join(map(str, (t, *p, group))) for t, p, group in FOUR])
def test_products_of_4_bits(type_, p, group, gated):
    n, cols, K = p
    gen = on_gpu("exact 4", type_, n, cols, K, group, gated)
    four_bits_are_exact(type_, n, cols, K, group, gated, whole(gen, (n, K)), gen, range(1, 8))
    if type_ == "f32":                                                # all bits of what enters as three numbers, times powers of two
        four_bits_are_exact(type_, n, cols, K, group, gated, one_of_a_row(gen, n, K), gen, (1, 2, 4, 6))


# a launch has 65535 blocks of rows, of 64 (fp32: 32) each; f_in shorter than 16 bytes goes by these blocks whatever the rows
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("type_,n,K", [("bf16", 65535 * 64 + 100, 5), ("f16", 2 * 65535 * 64 + 1, 3), ("f32", 65535 * 32 + 77, 3)])
def test_more_rows_than_a_launch_has_blocks_for(type_, n, K, gated):
    gen = on_gpu("blocks", type_, n, K, gated)
    R = None if gated else whole(gen, (n, 12)).to(TYPES[type_])
    four_bits_are_exact(type_, n, 12, K, 32, gated, whole(gen, (n, K)), gen, range(1, 8), R)


@pytest.mark.parametrize("type_", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("op", ["gated", "gated checkpoint", "linear checkpoint"])
@pytest.mark.parametrize("n,K,N", [(33, 64, 96), (515, 130, 201), (4099, 602, 1001), (1024, 1024, 512)])
def test_backward_products_are_those_of_the_dz_that_is_left(type_, op, n, K, N):
    """dX and dW are off from the products of the rounded dZ by the sums in 32 bits and their own rounding only."""
    g = lib()
    gen = gen_of("dz", type_, op, n, K, N)
    cols = 2 * N if op.startswith("gated") else N
    z, x = normal(gen, (n, cols), type_), normal(gen, (n, K), type_)
    W, dH = normal(gen, (K, cols), type_, K ** -0.5).cuda(), normal(gen, (n, N), type_).cuda()
    if "checkpoint" in op:
        (bx, x), (bz, _) = kept(x, type_, 0, 0), kept(z, type_, 0, 0)
        X, Z = bx.pair(), bz.pair()
    else:
        X, Z = x.cuda(), z.cuda()
    dZ, dX, dW = out(n, cols, type_), out(n, K, type_), out(K, cols, type_)
    if op.startswith("gated"):
        g.gcn_gated_backward(X, W, Z, dH, dZ.t, dX=dX.t, dW=dW.t, act=g.ACT_GELU)
    else:
        g.gcn_checkpoint_linear_backward(X, W, Z, dH, dZ.t, dX=dX.t, dW=dW.t, act=g.ACT_GELU)
    d, w, x = dZ.t.double(), W.double(), x.double().cuda()
    for t, a, b, terms in ((dX.t, d, w.t().contiguous(), cols), (dW.t, x.t().contiguous(), d, n)):
        ref, off = a @ b, (terms + 2) * EPS * (a.abs() @ b.abs())
        check(t, ref.cpu(), (off + UNIT[type_] * (ref.abs() + off) + TINY[type_]).cpu(), "dX" if t is dX.t else "dW")
