"""Every kernel of gated blocks of up to 32 rows, at the sizes that gated_few.py lists, against products in 64 bits and against sums that are exact."""
import pytest

torch = pytest.importorskip("torch")

from gated_few import FEW_GATED
from test_gpu_gated_tiles import by_types, names, test_gated_tiles as as_tiles
from test_gpu_linear_tiles import matrix
from test_gpu_operators import TYPES, gen_of, lib

pytestmark = pytest.mark.gpu

# (elements, rows, f_out, f_in), as the tiles' list has them
SIZES = [(p[0], None, *p[1:4], *p[4:]) for p in FEW_GATED]
CASES = by_types(SIZES)


@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("type_,p", CASES, ids=names(CASES))
def test_few_rows(type_, p, whole):
    as_tiles(type_, (None, whole, None, None, *p[-3:]))


@pytest.mark.parametrize("type_,p", CASES, ids=names(CASES))
def test_few_rows_of_whole_numbers(type_, p):
    """X of whole numbers up to 3 and weights of +-1 and +-2: every sum is exact in 32 bits, whatever its order (20003 x 6 is far below 2^24), so that a value of k left out or taken twice shows."""
    g = lib()
    n, N, K = p[-3:]
    gen = gen_of("whole numbers", type_, n, N, K)
    x = torch.randint(-3, 4, (n, K), generator=gen).double()
    w = (torch.randint(1, 3, (K, 2 * N), generator=gen) * (2 * torch.randint(0, 2, (K, 2 * N), generator=gen) - 1)).double()
    X, W = matrix(n, K, type_, False, x), matrix(K, 2 * N, type_, False, w)
    H, Z = matrix(n, N, type_, False), matrix(n, 2 * N, type_, False)
    g.gcn_gated_forward(X.t, W.t, H.t, act=g.ACT_NONE, Z=Z.t)
    z = (x.cuda() @ w.cuda()).float()
    assert torch.equal(Z.t, z.to(TYPES[type_]))
    assert torch.equal(H.t, (z[:, :N] * z[:, N:]).to(TYPES[type_]))
    assert H.outside_is_untouched() and Z.outside_is_untouched()
