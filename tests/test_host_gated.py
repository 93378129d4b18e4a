"""What gated blocks, checkpoints and weights in 4 bits refuse: decided on the host, before anything is launched or read, so without a GPU."""
import pytest

import paper_2005_03300_amd as g

BADARG, RANGE = -1, -2
P = [0x10000000 * (i + 1) for i in range(12)]          # places that nothing is read from
FAR = (1 << 31) - 1


def refused(rc, want, text=""):
    said = g.lib().gcn_last_error().decode()
    assert rc == want and text in said, (rc, said)


def gated_forward(n=8, fi=16, fo=8, type_=1, X=P[0], ldx=16, W=P[1], ldw=16, bias=P[2], act=3, Z=P[3], ldz=16, H=P[4], ldh=8):
    return g.lib().gcn_gated_forward(n, fi, fo, type_, X, ldx, W, ldw, bias, act, Z, ldz, H, ldh, 0)


def test_gated_forward():
    for name in ("X", "W", "H"):
        refused(gated_forward(**{name: 0}), BADARG, "NULL")
    for bad in (dict(n=0), dict(fi=0), dict(fo=-1)):
        refused(gated_forward(**bad), BADARG, "positive")
    refused(gated_forward(type_=3), BADARG, "element type")
    refused(gated_forward(act=4), BADARG, "activation")
    for name, low in (("ldx", 15), ("ldw", 15), ("ldz", 15), ("ldh", 7)):
        refused(gated_forward(**{name: low}), BADARG, "leading dimension")
    refused(gated_forward(n=1, fi=(1 << 27) + 1, ldx=FAR), RANGE)
    refused(gated_forward(n=1, fo=(1 << 26) + 1, ldw=FAR, ldz=FAR, ldh=FAR), RANGE)
    for bad in (dict(H=P[0]), dict(H=P[1] + 32), dict(H=P[2] + 60), dict(Z=P[0] + 30), dict(Z=P[1]), dict(Z=P[2] + 2), dict(Z=P[4] - 14)):
        refused(gated_forward(**bad), BADARG, "overlaps")


def gated_backward(n=8, fi=16, fo=8, type_=1, X=P[0], ldx=16, xs=0, ldxs=0, W=P[1], ldw=16, Z=P[2], ldz=16, zs=0, ldzs=0, dH=P[3], lddh=8, act=3, dZ=P[4], lddz=16, dX=P[5], lddx=16, dW=P[6],
                   lddw=16, db=P[7], H=P[8], ldh=8):
    return g.lib().gcn_gated_backward(n, fi, fo, type_, X, ldx, xs, ldxs, W, ldw, Z, ldz, zs, ldzs, dH, lddh, act, dZ, lddz, dX, lddx, dW, lddw, db, H, ldh, 0)


def test_gated_backward():
    for name in ("X", "W", "Z", "dH"):
        refused(gated_backward(**{name: 0}), BADARG, "NULL")
    refused(gated_backward(dZ=0), BADARG, "workspace")
    for bad in (dict(n=0), dict(fi=0), dict(fo=-1)):
        refused(gated_backward(**bad), BADARG, "positive")
    refused(gated_backward(type_=-1), BADARG, "element type")
    refused(gated_backward(act=9), BADARG, "activation")
    for name, low in (("ldx", 15), ("ldw", 15), ("ldz", 15), ("lddh", 7), ("lddz", 15), ("lddx", 15), ("lddw", 15), ("ldh", 7)):
        refused(gated_backward(**{name: low}), BADARG, "leading dimension")
    refused(gated_backward(xs=P[9], ldxs=0), BADARG, "leading dimension")
    refused(gated_backward(zs=P[9], ldzs=0), BADARG, "leading dimension")
    refused(gated_backward(n=1, fo=(1 << 26) + 1, ldw=FAR, ldz=FAR, lddh=FAR, lddz=FAR, lddw=FAR, ldh=FAR), RANGE)
    scales = dict(xs=P[9], ldxs=1, zs=P[10], ldzs=1)
    for bad in (dict(dX=P[0]), dict(dW=P[1]), dict(db=P[3] + 8), dict(H=P[4]), dict(dX=P[4] + 16), dict(dZ=P[3]), dict(dZ=P[2] + 2), dict(H=P[3] + 2),
                dict(scales, dZ=P[2]), dict(scales, dZ=P[9]), dict(scales, H=P[10] + 14), dict(scales, dX=P[9] - 2)):
        refused(gated_backward(**bad), BADARG, "overlaps")


def pack(f, n=4, width=100, type_=1, X=P[0], ldx=100, C=P[1], ldc=100, S=P[2], lds=2):
    L = g.lib()
    if f == "pack":
        return L.gcn_checkpoint_pack(n, width, type_, X, ldx, C, ldc, S, lds, 0)
    return L.gcn_checkpoint_unpack(n, width, type_, C, ldc, S, lds, X, ldx, 0)


@pytest.mark.parametrize("f", ["pack", "unpack"])
def test_checkpoint_pack(f):
    for name in ("X", "C", "S"):
        refused(pack(f, **{name: 0}), BADARG, "NULL")
    refused(pack(f, n=0), BADARG, "positive")
    refused(pack(f, width=0), BADARG, "positive")
    refused(pack(f, type_=7), BADARG, "element type")
    for name, low in (("ldx", 99), ("ldc", 99), ("lds", 1)):
        refused(pack(f, **{name: low}), BADARG, "leading dimension")
    refused(pack(f, n=1, width=(1 << 27) + 1, ldx=FAR, ldc=FAR, lds=FAR), RANGE)
    for bad in (dict(C=P[0]), dict(S=P[0] + 798), dict(S=P[1] + 399), dict(C=P[0] - 399)):
        refused(pack(f, **bad), BADARG, "overlaps")


def linear_backward(n=8, fi=16, fo=8, type_=1, X=P[0], ldx=16, xs=P[9], ldxs=1, W=P[1], ldw=8, Z=P[2], ldz=8, zs=P[10], ldzs=1, dY=P[3], lddy=8, act=3, dZ=P[4], lddz=8, dX=P[5], lddx=16,
                    dW=P[6], lddw=8, db=P[7], dR=P[8], lddr=8):
    return g.lib().gcn_checkpoint_linear_backward(n, fi, fo, type_, X, ldx, xs, ldxs, W, ldw, Z, ldz, zs, ldzs, dY, lddy, act, 0.5, dZ, lddz, dX, lddx, dW, lddw, db, dR, lddr, 0)


def test_checkpoint_linear_backward():
    for name in ("X", "W", "dY"):
        refused(linear_backward(**{name: 0}), BADARG, "NULL")
    refused(linear_backward(Z=0), BADARG, "needs Z")
    refused(linear_backward(dZ=0), BADARG, "workspace")
    refused(linear_backward(n=-1), BADARG, "positive")
    refused(linear_backward(type_=3), BADARG, "element type")
    refused(linear_backward(act=-1), BADARG, "activation")
    for name, low in (("ldx", 15), ("ldxs", 0), ("ldw", 7), ("ldz", 7), ("ldzs", 0), ("lddy", 7), ("lddz", 7), ("lddx", 15), ("lddw", 7), ("lddr", 7)):
        refused(linear_backward(**{name: low}), BADARG, "leading dimension")
    refused(linear_backward(n=1, fo=(1 << 27) + 1, ldw=FAR, ldz=FAR, ldzs=FAR, lddy=FAR, lddz=FAR, lddw=FAR, lddr=FAR), RANGE)
    for bad in (dict(dZ=P[2]), dict(dZ=P[10]), dict(dX=P[9]), dict(dX=P[0]), dict(dW=P[1]), dict(dR=P[3] + 2), dict(db=P[8]), dict(act=0, dR=P[3])):
        refused(linear_backward(**bad), BADARG, "overlaps")


def layout(f, K=100, cols=40, type_=1, W=P[0], ldw=40, group=32, Q=P[1], ldq=40, S=P[2], lds=40):
    L = g.lib()
    if f == "pack":
        return L.gcn_linear4_pack(K, cols, type_, W, ldw, group, Q, ldq, S, lds, 0)
    return L.gcn_linear4_unpack(K, cols, type_, Q, ldq, S, lds, group, W, ldw, 0)


@pytest.mark.parametrize("f", ["pack", "unpack"])
def test_linear4_layout(f):
    for name in ("W", "Q", "S"):
        refused(layout(f, **{name: 0}), BADARG, "NULL")
    for bad in (dict(K=0), dict(cols=0)):
        refused(layout(f, **bad), BADARG, "positive")
    for group in (0, 16, 48, 256, -32):
        refused(layout(f, group=group), BADARG, "groups")
    refused(layout(f, type_=3), BADARG, "element type")
    for name in ("ldw", "ldq", "lds"):
        refused(layout(f, **{name: 39}), BADARG, "leading dimension")
    refused(layout(f, K=(1 << 27) + 1), RANGE)
    refused(layout(f, K=1, cols=(1 << 27) + 1, ldw=FAR, ldq=FAR, lds=FAR), RANGE)
    for bad in (dict(Q=P[0]), dict(S=P[0] + 7998), dict(S=P[1] + 13 * 160 - 2)):
        refused(layout(f, **bad), BADARG, "overlaps")


def forward4(n=4, K=100, N=40, type_=1, X=P[0], ldx=100, Q=P[1], ldq=80, S=P[2], lds=80, group=64, gated=1, bias=P[3], act=3, R=P[4], ldr=40, Y=P[5], ldy=40):
    return g.lib().gcn_linear4_forward(n, K, N, type_, X, ldx, Q, ldq, S, lds, group, gated, bias, act, R, ldr, 1.0, Y, ldy, 0)


def test_linear4_forward():
    for name in ("X", "Q", "S", "Y"):
        refused(forward4(**{name: 0}), BADARG, "NULL")
    for bad in (dict(n=0), dict(K=0), dict(N=0)):
        refused(forward4(**bad), BADARG, "positive")
    refused(forward4(group=96), BADARG, "groups")
    refused(forward4(type_=3), BADARG, "element type")
    refused(forward4(act=4), BADARG, "activation")
    for name, low in (("ldx", 99), ("ldq", 79), ("lds", 79), ("ldr", 39), ("ldy", 39)):
        refused(forward4(**{name: low}), BADARG, "leading dimension")
    refused(forward4(n=1, K=(1 << 27) + 1, ldx=FAR), RANGE)
    refused(forward4(n=1, N=(1 << 26) + 1, ldq=FAR, lds=FAR, ldr=FAR, ldy=FAR), RANGE)
    for bad in (dict(Y=P[0]), dict(Y=P[1]), dict(Y=P[2]), dict(Y=P[3]), dict(Y=P[4] + 2), dict(Y=P[4], ldy=41)):
        refused(forward4(**bad), BADARG, "overlaps")


def test_binding_looks_at_shapes():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 100)
    with pytest.raises(AssertionError):
        g.gcn_checkpoint_pack(x, torch.zeros(4, 100, dtype=torch.int8), torch.zeros(4, 2, dtype=torch.bfloat16))
    with pytest.raises(AssertionError):
        g.gcn_linear4_pack(x, torch.zeros(1, 100, dtype=torch.int32), torch.zeros(1, 100, dtype=torch.bfloat16), group=0)


def test_sizes_take_the_kernels_that_they_stand_for(tmp_path):
    """The lists that the GPU tests go through hold every kernel, and their sizes choose it."""
    from gated_tiles import FEW4, GATED, TILES4
    from test_host_parts import run_cpp
    calls = "".join(f"gated({M}, {2 * N}, {K}, {int(t == 'f32')}, {int(w)});" for t, w, _, _, M, N, K in GATED)
    calls += "".join(f"few({M}, {N}, {K}, {int(t == 'f32')});" for t, _, _, _, M, N, K in FEW4)
    calls += "".join(f"tiles({M}, {N}, {K}, {int(t == 'f32')});" for t, _, M, N, K in TILES4)
    r = run_cpp(tmp_path, """
        #include <cstdio>
        #include "launch_rules.h"
        using namespace gcn;
        void gated(int64_t M, int64_t N, int64_t K, int fp32, int direct) {
            const TileChoice c = choose_tiles(M, N, K, fp32, direct, 256);
            printf("%%d %%d\\n", c.edge, c.splits);
        }
        void few(int64_t M, int64_t N, int64_t K, int fp32) {
            const Few4 f = few4_choice(M, N, K, fp32, 256);
            printf("%%d %%d %%d\\n", f.rows, f.columns, (int)f.splits);
        }
        void tiles(int64_t M, int64_t N, int64_t K, int fp32) {
            printf("%%d %%d\\n", few4_choice(M, N, K, fp32, 256).rows, splits_of_4((M + 127) / 128 * ((N + 127) / 128), M * N, K, fp32, 256));
        }
        int main() { %s }
    """ % calls)
    got = [tuple(map(int, line.split())) for line in r.stdout.splitlines()]
    want = [p[2:4] for p in GATED] + [p[1:4] for p in FEW4] + [(0, p[1]) for p in TILES4]
    assert got == want, [(g_, w_) for g_, w_ in zip(got, want) if g_ != w_]
    assert {(p[0], p[1], p[2], p[3] > 1) for p in GATED} == {("16", w, e, s) for w in (False, True) for e in (256, 128, 64) for s in (False, True)} | {
        ("f32", False, e, s) for e in (128, 64) for s in (False, True)}
    assert {(p[0], p[1], p[2]) for p in FEW4} == {("16", r, c) for r in (1, 2, 4) for c in (1, 2, 4, 8) if (r, c) != (4, 8)} | {("f32", 1, c) for c in (1, 4, 8)} | {
        ("f32", 2, c) for c in (1, 2, 4)}
    # k shorter than 16 bytes, which tiles do not take: any number of rows goes the other way
    r = run_cpp(tmp_path, """
        #include <cstdio>
        #include <initializer_list>
        #include "launch_rules.h"
        int main() {
            for (int64_t M : {1, 65, 20000, 100000000})
                for (int64_t cols : {1, 300, 1 << 27})
                    for (int64_t K : {1, 3, 7, 8, 100, 1 << 27})
                        for (int fp32 : {0, 1}) {
                            const gcn::Few4 f = gcn::few4_choice(M, cols, K, fp32, 256);
                            const bool tiles = K >= (fp32 ? 4 : 8);
                            if (f.rows == 0 ? !tiles : f.columns < 1 || f.splits < 1) return printf("%lld %lld %lld\\n", (long long)M, (long long)cols, (long long)K), 1;
                        }
        }
    """)
    assert r.returncode == 0, r.stdout
    assert {p[0] for p in FEW4 if p[3] > 1} == {p[0] for p in TILES4 if p[1] > 1} == {"16", "f32"}
