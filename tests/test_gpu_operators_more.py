"""The operators of residual networks at the ends of what they take: magnitudes, widths, places of operands, tiles.

Tolerances are derived as in test_gpu_operators.py."""
import math

import pytest

torch = pytest.importorskip("torch")

from test_gpu_operators import ALL, EPS, TINY, TYPES, UNIT, check, code, gen_of, lib, normal

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
