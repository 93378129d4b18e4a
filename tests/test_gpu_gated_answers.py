"""What the example's student of gated blocks keeps between its passes, and its answers from weights in 4 bits."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_gated_student import example
from test_gpu_operators import TYPES

pytestmark = pytest.mark.gpu


def student(m, n, type_, blocks=2, width=64, f=24, classes=8):
    s = m.Student(n, f, width, classes, blocks, TYPES[type_], seed=3, gated=True)
    gen = torch.Generator(device="cuda").manual_seed(5)
    for v in s.vec.values():                                          # biases and weights of norms that show where one is left out
        v += 0.5 * torch.randn(v.shape, generator=gen, device="cuda")
    return s, torch.randn(n, f, generator=gen, device="cuda").to(TYPES[type_])


def test_blocks_inputs_are_kept_once():
    """In 8 bits, for every block of its own; the rows themselves are one block's at a time."""
    s, _ = student(example(), 100, "bf16", blocks=3)
    assert len({t.data_ptr() for t in s.H}) == len({t.data_ptr() for t in s.Z1}) == len({t.data_ptr() for t in s.Y1}) == 1
    assert len({c.data_ptr() for c, _ in s.H8}) == len({c.data_ptr() for c, _ in s.Z8}) == 3


def test_answers_write_no_checkpoints():
    s, P = student(example(), 100, "bf16")
    for c, t in s.H8 + s.Z8:
        c.fill_(77)
        t.fill_(3.0)
    logits = s.forward(P).clone()
    assert all(bool((c == 77).all()) and bool((t == 3.0).all()) for c, t in s.H8 + s.Z8)
    assert torch.equal(s.forward(P, keep=True), logits)
    assert not any(bool((c == 77).all()) for c, _ in s.H8 + s.Z8)


# In 32 bits a product of K <= 128 normal numbers is off by (K + 2) 2^-24 of its terms' absolute sum, which is 0.64 sqrt(K) times the result's size: 5.6e-5 of it.  Eight products one after another
# (one in front, three of each block, one behind), each error at most doubled by the norm that follows: 9e-4.  Types of 16 bits round each of about twelve results on the way, half a step each, at most
# doubled as well: 24 2^-8 and 24 2^-11.
@pytest.mark.parametrize("type_,tol", [("f32", 1e-3), ("bf16", 24 * 2.0 ** -8), ("f16", 24 * 2.0 ** -11)])
def test_answers_from_4_bits(type_, tol):
    """Against a forward pass in 64 bits with the weights that the codes stand for, for many rows and for one."""
    m = example()
    g = m.g
    s, P = student(m, 300, type_)
    four = m.FourBits(s)
    W = {}
    for k, (Q, S) in four.W.items():
        w = torch.empty(s.master[k].shape, device="cuda")             # a place times its scale has ten bits: exact
        g.gcn_linear4_unpack(Q, S, w, group=four.group)
        W[k] = w.double()
    v = {k: t.double() for k, t in s.vec.items()}

    def norm(x, w):
        return x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-5) * w
    X = P.double() @ W["in"] + v["in.b"]
    H = norm(X, v["norm0"])
    for l in range(s.blocks):
        gate, up = (H @ W[f"{l}.W1"] + v[f"{l}.b1"]).chunk(2, 1)
        U = (torch.nn.functional.silu(gate) * up) @ W[f"{l}.W2"] + v[f"{l}.b2"]
        X = X + v[f"{l}.scale"] * torch.sigmoid(H @ W[f"{l}.G"]) * norm(U, v[f"{l}.post"])
        H = norm(X, v[f"norm{l + 1}"])
    want = H @ W["out"]
    got = four.answer(P).double()
    size = want.norm(dim=1).mean()
    assert float((got - want).norm()) <= tol * float(want.norm())
    for i in (0, 123):
        one = four.answer(P[i:i + 1].contiguous()).double()
        assert float((one - want[i:i + 1]).norm()) <= 2 * tol * float(size)
    if type_ == "f32":                                                # (the student's own weights are others, whose answers would not do)
        assert float((s.forward(P).double() - want).norm()) > 10 * tol * float(want.norm())
