"""A graph network as teacher, and a student without a graph trained from the teacher's largest logits.

The teacher is the two-layer GCN of the tiny workload (4096 vertices, 64 -> 16 -> 8), trained with gcn_epoch.  The student sees each
vertex by itself: its features aggregated over one step and over two (A^T H0 and A^T A^T H0, two calls of gcn_spmm, computed
once) pass through residual blocks

    X' = X + scale * sigmoid(H G) * N(act(H W1 + b1) W2 + b2),   H' = N(X')

and a last linear layer; its loss is gcn_distill against the teacher's k largest logits per vertex and the labels.  Answering for a
vertex afterwards needs neither the graph nor the teacher.

    python examples/distill_student.py [--type bf16|f16|f32] [--blocks 2] [--width 128] [--steps 200]
"""
from __future__ import annotations

import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch

import paper_2005_03300_amd as g
import synth

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def teacher(steps: int = 600, lr: float = 30.0):
    """(logits of all vertices, labels, aggregated features): a GCN trained on labels that the features aggregated over two steps give (the class is
    the largest of eight random projections, each about its mean)."""
    w = synth.CONFIGS[1]
    n, src, dst = synth.make_graph(w)
    H0, _, Ws = synth.make_model_inputs(w)
    dims = list(w.dims)
    a = g.gcn_csr_create(n, torch.from_numpy(src).cuda(), torch.from_numpy(dst).cuda(),
                         g.SYMMETRISE | g.ADD_SELF_LOOPS | g.NORM_SYM | g.BUILD_TRANSPOSE)
    H0 = torch.from_numpy(H0).cuda()
    one, two = torch.empty_like(H0), torch.empty_like(H0)
    g.gcn_spmm(a, 1, H0, one)
    g.gcn_spmm(a, 1, one, two)
    P = torch.cat([one, two], 1)
    gen = torch.Generator(device="cuda").manual_seed(3)
    score = two @ torch.randn(dims[0], dims[-1], generator=gen, device="cuda")
    labels = ((score - score.mean(0)) / score.std(0)).argmax(1).int()
    W = [torch.from_numpy(x).cuda() for x in Ws]
    Y = [torch.empty_like(x) for x in W]
    loss = torch.empty(1, device="cuda")
    work = torch.empty(g.gcn_epoch_workspace_bytes(n, dims), dtype=torch.uint8, device="cuda")
    for _ in range(steps):
        g.gcn_epoch(a, dims, H0, labels, W, Y, lr, loss, work)
    Z, H, T = (torch.empty(n, dims[1], device="cuda") for _ in range(3))
    g.gcn_layer_forward(a, H0, W[0], Z, H, T, act=g.ACT_RELU)
    logits, T = torch.empty(n, dims[2], device="cuda"), torch.empty(n, max(dims[1:]), device="cuda")
    g.gcn_layer_forward(a, H, W[1], logits, None, T.view(-1)[:n * dims[2]].view(n, dims[2]), order=g.ORDER_GEMM_FIRST, act=g.ACT_NONE)
    torch.cuda.synchronize()
    a.close()
    return logits, labels, P


class Student:
    """Weights in the element type with fp32 copies that the steps are taken on; buffers for one training step over n rows."""

    def __init__(self, n: int, f_in: int, width: int, classes: int, blocks: int, dtype, seed: int = 0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.dtype, self.blocks, self.n = dtype, blocks, n

        def glorot(i, o):
            return torch.randn(i, o, generator=gen, device="cuda") * (2.0 / (i + o)) ** 0.5
        self.master = {"in": glorot(f_in, width), "out": glorot(width, classes)}
        self.vec = {"in.b": torch.zeros(width, device="cuda"), "norm0": torch.ones(width, device="cuda")}
        for l in range(blocks):
            self.master.update({f"{l}.W1": glorot(width, 2 * width), f"{l}.W2": glorot(2 * width, width), f"{l}.G": glorot(width, width)})
            self.vec.update({f"{l}.b1": torch.zeros(2 * width, device="cuda"), f"{l}.b2": torch.zeros(width, device="cuda"),
                             f"{l}.scale": torch.full((width,), 0.5, device="cuda"), f"{l}.post": torch.ones(width, device="cuda"),
                             f"norm{l + 1}": torch.ones(width, device="cuda")})
        self.W = {k: v.to(dtype) for k, v in self.master.items()}
        self.dW = {k: torch.empty_like(v) for k, v in self.W.items()}
        self.dvec = {k: torch.empty_like(v) for k, v in self.vec.items()}
        e = lambda cols: torch.empty(n, cols, dtype=dtype, device="cuda")
        rows = lambda: torch.empty(n, 4, device="cuda")
        self.X, self.H, self.st = [e(width) for _ in range(blocks + 1)], [e(width) for _ in range(blocks + 1)], [rows() for _ in range(blocks + 1)]
        self.Z1, self.Y1 = [e(2 * width) for _ in range(blocks)], [e(2 * width) for _ in range(blocks)]
        self.U, self.A = [e(width) for _ in range(blocks)], [e(width) for _ in range(blocks)]
        self.logits, self.G = e(classes), e(classes)
        self.dX, self.dH, self.dH2, self.dU, self.dA = (e(width) for _ in range(5))
        self.dY1, self.dZ1 = e(2 * width), e(2 * width)
        self.loss = torch.empty(1, device="cuda")
        self.momentum = {}

    def forward(self, P):
        W, v = self.W, self.vec
        g.gcn_linear_forward(P, W["in"], self.X[0], bias=v["in.b"])
        g.gcn_block_norm_forward(self.X[0], H=self.H[0], w_pre=v["norm0"], stats=self.st[0])
        for l in range(self.blocks):
            H = self.H[l]
            g.gcn_linear_forward(H, W[f"{l}.W1"], self.Y1[l], bias=v[f"{l}.b1"], act=g.ACT_GELU, Z=self.Z1[l])
            g.gcn_linear_forward(self.Y1[l], W[f"{l}.W2"], self.U[l], bias=v[f"{l}.b2"])
            g.gcn_linear_forward(H, W[f"{l}.G"], self.A[l])
            g.gcn_block_norm_forward(self.X[l], self.U[l], self.X[l + 1], self.H[l + 1], w_pre=v[f"norm{l + 1}"], A=self.A[l],
                                     scale=v[f"{l}.scale"], w_post=v[f"{l}.post"], stats=self.st[l + 1])
        g.gcn_linear_forward(self.H[-1], W["out"], self.logits)
        return self.logits

    def step(self, P, top, t, labels, lr: float, temperature: float = 2.0):
        """One step of gradient descent over all rows; returns the loss (on the device)."""
        W, dW, v, dv = self.W, self.dW, self.vec, self.dvec
        self.forward(P)
        # half-precision gradients of a mean over many rows would be lost below the type's smallest numbers: they are carried n times as large
        g.gcn_distill(self.logits, top, t, self.loss, self.G, labels=labels, temperature=temperature, w_teacher=0.7, w_label=0.3,
                      grad_scale=float(self.n))
        g.gcn_linear_backward(self.H[-1], W["out"], None, self.G, dX=self.dH, dW=dW["out"])
        dXout = None
        for l in reversed(range(self.blocks)):
            g.gcn_block_norm_backward(self.U[l], self.X[l + 1], self.st[l + 1], dXout, self.dH, self.dX, self.dU, w_pre=v[f"norm{l + 1}"],
                                      A=self.A[l], dA=self.dA, scale=v[f"{l}.scale"], w_post=v[f"{l}.post"], dscale=dv[f"{l}.scale"],
                                      dw_post=dv[f"{l}.post"], dw_pre=dv[f"norm{l + 1}"])
            dXout = self.dX
            g.gcn_linear_backward(self.Y1[l], W[f"{l}.W2"], None, self.dU, dX=self.dY1, dW=dW[f"{l}.W2"], dbias=dv[f"{l}.b2"])
            g.gcn_linear_backward(self.H[l], W[f"{l}.W1"], self.Z1[l], self.dY1, self.dZ1, dX=self.dH, dW=dW[f"{l}.W1"],
                                  dbias=dv[f"{l}.b1"], act=g.ACT_GELU)
            g.gcn_linear_backward(self.H[l], W[f"{l}.G"], None, self.dA, dX=self.dH2, dW=dW[f"{l}.G"])
            self.dH += self.dH2
        g.gcn_block_norm_backward(None, self.X[0], self.st[0], dXout, self.dH, self.dX, w_pre=v["norm0"], dw_pre=dv["norm0"])
        g.gcn_linear_backward(P, None, None, self.dX, dW=dW["in"], dbias=dv["in.b"])
        for k, m in self.master.items():
            m -= self.pace(k, lr, dW[k])
            W[k].copy_(m)
        for k, x in v.items():
            x -= self.pace(k, lr, dv[k])
        return self.loss

    def pace(self, k, lr: float, gradient):
        """Gradient descent with momentum."""
        b = self.momentum.setdefault(k, torch.zeros_like(gradient, dtype=torch.float32))
        b.mul_(0.9).add_(gradient, alpha=1.0 / self.n)
        return lr * b


def train(dtype: str = "bf16", blocks: int = 2, width: int = 128, steps: int = 200, k: int = 4, lr: float = 0.1, say=print):
    """Trains a student; returns (first loss, last loss, share of vertices on which it agrees with the teacher)."""
    logits, labels, P = teacher()
    dt = TYPES[dtype]
    t, top = logits.topk(k, dim=1)
    t, top, P = t.to(dt).contiguous(), top.int().contiguous(), ((P - P.mean(0)) / P.std(0)).to(dt)
    s = Student(P.shape[0], P.shape[1], width, logits.shape[1], blocks, dt)
    first = None
    for i in range(steps):
        loss = s.step(P, top, t, labels, lr * (1.0 - i / steps))
        if i % max(1, steps // 8) == 0 or i == steps - 1:
            say(f"step {i:4d}  loss {loss.item():.4f}")
        first = loss.item() if first is None else first
    agree = (s.forward(P).argmax(1) == logits.argmax(1)).float().mean().item()
    one = torch.empty(1, logits.shape[1], dtype=dt, device="cuda")         # a single vertex, as in serving
    alone = Student(1, P.shape[1], width, logits.shape[1], blocks, dt)
    alone.W, alone.vec = s.W, s.vec
    one.copy_(alone.forward(P[:1].contiguous()))
    say(f"agrees with the teacher on {100 * agree:.1f} % of the vertices; vertex 0 alone: class {one.argmax().item()}")
    return first, s.loss.item(), agree


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--type", default="bf16", choices=sorted(TYPES))
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--width", type=int, default=128)
    ap.add_argument("--steps", type=int, default=200)
    args = ap.parse_args()
    train(args.type, args.blocks, args.width, args.steps)
