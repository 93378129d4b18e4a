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
