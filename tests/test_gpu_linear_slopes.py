"""dZ, dR and the bias's gradient of linear layers, at sizes that take each kernel of theirs, against 64 bits; and in the place of what they are made of.

Tolerances are derived as in test_gpu_operators.py."""
import pytest

torch = pytest.importorskip("torch")

from linear_slopes import SLOPES
from test_gpu_gated_tiles import by_types, names
from test_gpu_operators import ACTS, EPS, TINY, UNIT, Strided, check, code, gen_of, lib, normal, out, slope64

pytestmark = pytest.mark.gpu

CASES = by_types(SLOPES)


@pytest.mark.parametrize("pad,skip", [(0, 0), (3, 1)])
@pytest.mark.parametrize("type_,p", CASES, ids=names(CASES))
def test_slopes(type_, p, pad, skip):
    g = lib()
    n, N = p[-2:]
    act = ACTS[(n + N + pad) % 4]
    gen = gen_of("slopes", type_, n, N, pad)
    z, dy, rho, u = normal(gen, (n, N), type_), normal(gen, (n, N), type_), -0.75, UNIT[type_]
    Z, dY, dZ, dR = Strided(n, N, type_, pad, skip, z), Strided(n, N, type_, pad, skip, dy), out(n, N, type_, pad, skip), out(n, N, type_, pad, skip)
    db = torch.empty(N, device="cuda")
    curved = act != "none"
    args = dict(act=code(g, act), rho=rho)
    g.gcn_linear_backward(None, None, Z.t if curved else None, dY.t, dZ.t, dbias=db, dR=dR.t, **args)
    z, dy = z.double(), dy.double()
    dz = dy * slope64(z, act) if curved else dy
    near = 10 * EPS * (z.abs() + 2) * dy.abs() if curved else torch.zeros_like(dy)
    if curved:
        check(dZ.t, dz, near + u * (dz.abs() + near) + TINY[type_], "dZ")
    check(dR.t, rho * dy, (EPS + u) * (rho * dy).abs() + TINY[type_], "dR")
    check(db, dz.sum(0), near.sum(0) + (n + 2) * EPS * (dz.abs() + near).sum(0) + 1e-37, "dbias")
    assert dZ.outside_is_untouched() and dR.outside_is_untouched()
    # each by itself, and in place, has the same bits
    again = torch.empty_like(db)
    g.gcn_linear_backward(None, None, Z.t if curved else None, dY.t, dbias=again, **args)
    assert torch.equal(again, db)
    if curved:
        z_place, y_place = Strided(n, N, type_, pad, skip, Z.t), Strided(n, N, type_, pad, skip, dY.t)
        g.gcn_linear_backward(None, None, z_place.t, y_place.t, z_place.t, dbias=again, dR=y_place.t, **args)
        assert torch.equal(z_place.t, dZ.t) and torch.equal(y_place.t, dR.t) and torch.equal(again, db)
        y_place = Strided(n, N, type_, pad, skip, dY.t)
        g.gcn_linear_backward(None, None, Z.t, y_place.t, y_place.t, **args)
        assert torch.equal(y_place.t, dZ.t)
        for b in (z_place, y_place):
            assert b.outside_is_untouched()
