"""The example's student of gated blocks, which trains from checkpoints in 8 bits and answers from weights in 4: that it runs, and its gradients."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("distill_student", os.path.join(ROOT, "examples", "distill_student.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("type_", ["f32", "bf16", "f16"])
def test_gated_student_runs(type_):
    lines = []
    first, last, agree = example().train(type_, blocks=2, width=64, steps=6, say=lines.append, gated=True)
    assert all(x == x and abs(x) < float("inf") for x in (first, last, agree))
    assert any("vertex 0 alone" in x for x in lines) and any("4 bits" in x for x in lines)


def test_gated_student_gradients():
    """All gradients of one step against autograd in 64 bits: fp32 rows, so that what is left is that the first layer's input and argument are kept in 8 bits, off by 1/254 of the largest of 64
    neighbours at most, or about a hundredth of their size."""
    m = example()
    g = m.g
    n, f, width, classes, k = 50, 24, 64, 8, 3
    s = m.Student(n, f, width, classes, 2, torch.float32, seed=3, gated=True)
    gen = torch.Generator(device="cuda").manual_seed(4)
    for name, v in s.vec.items():
        v += 0.1 * torch.randn(v.shape, generator=gen, device="cuda")
    P = torch.randn(n, f, generator=gen, device="cuda")
    t, top = torch.randn(n, classes, generator=gen, device="cuda").topk(k, dim=1)
    labels = torch.randint(classes, (n,), generator=gen, device="cuda", dtype=torch.int32)
    W = {a: b.double().requires_grad_() for a, b in s.W.items()}
    v = {a: b.double().requires_grad_() for a, b in s.vec.items()}

    def norm(x, w):
        return x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-5) * w
    X = P.double() @ W["in"] + v["in.b"]
    H = norm(X, v["norm0"])
    for l in range(2):
        gate, up = (H @ W[f"{l}.W1"] + v[f"{l}.b1"]).split(2 * width, 1)
        U = (torch.nn.functional.silu(gate) * up) @ W[f"{l}.W2"] + v[f"{l}.b2"]
        X = X + v[f"{l}.scale"] * torch.sigmoid(H @ W[f"{l}.G"]) * norm(U, v[f"{l}.post"])
        H = norm(X, v[f"norm{l + 1}"])
    z = H @ W["out"]
    T = 2.0
    p = torch.softmax(t.double() / T, 1)
    logq = torch.log_softmax(z / T, 1).gather(1, top)
    loss = 0.7 * T * T * (p * (p.log() - logq)).sum() + 0.3 * torch.nn.functional.cross_entropy(z, labels.long(), reduction="sum")
    want = dict(zip([*W, *v], torch.autograd.grad(loss, [*W.values(), *v.values()])))
    s.step(P, top.int().contiguous(), t.contiguous(), labels, lr=0.0, temperature=T)
    got = {**s.dW, **s.dvec}
    assert abs(s.loss.item() * n - loss.item()) < 1e-4 * abs(loss.item())
    for name, ref in want.items():
        off = float((got[name].double() - ref).norm() / ref.norm())
        assert off < 0.03, (name, off)
