"""The rule that gives gated blocks of few rows their strips and shares, by itself."""
from gated_few import FEW_GATED
from test_host_parts import run_cpp

CUS = 256


def choices(tmp_path, sizes):
    """(columns of a lane, shares) for each (fp32, rows, f_out, f_in)."""
    r = run_cpp(tmp_path, """
        #include <cstdio>
        #include "launch_rules.h"
        static void size(int fp32, int64_t M, int64_t N, int64_t K) {
            const gcn::FewGated f = gcn::few_gated_choice(M, N, K, fp32, %d);
            printf("%%d %%d\\n", f.columns, f.splits);
        }
        int main() { %s }
    """ % (CUS, "".join(f"size({int(f)}, {M}, {N}, {K});" for f, M, N, K in sizes)))
    return [tuple(map(int, line.split())) for line in r.stdout.splitlines()]


def test_sizes_take_the_kernels_that_they_stand_for(tmp_path):
    got = choices(tmp_path, [(p[0] == "f32", *p[4:]) for p in FEW_GATED])
    assert got == [p[2:4] for p in FEW_GATED], [(p, c) for p, c in zip(FEW_GATED, got) if p[2:4] != c]
    every = {("16", 1, c) for c in (1, 2, 4, 8)} | {("16", 2, c) for c in (1, 2, 4)} | {("f32", r, c) for r in (1, 2) for c in (1, 2, 4)}
    for shared in (False, True):
        assert {p[:3] for p in FEW_GATED if (p[3] > 1) == shared} == every


def test_no_size_leaves_compute_units_idle_that_its_neighbours_use(tmp_path):
    """Where k is long and strips alone would leave near half of the compute units idle, the sum is shared (shares grow by a half at most from two on, so that two thirds of the units have work); and neighbours
    take the same strips, or the next, never a shape of their own."""
    sizes = [(fp32, M, N, 8192) for fp32 in (False, True) for M in (1, 16, 24) for N in range(1024, 16385, 8)]
    got = choices(tmp_path, sizes)
    for (fp32, M, N, K), (columns, shares) in zip(sizes, got):
        strips = -(-N // (8 * columns))
        steps = -(-K // (256 if fp32 else 512))
        taken = strips * -(-steps // -(-steps // shares))
        rounds = -(-taken // CUS)
        assert taken / (rounds * CUS) > 0.6, (fp32, M, N, columns, shares)
    sizes = [(False, 1, N, 1000) for N in range(8000, 8400)]
    assert {c for c, _ in choices(tmp_path, sizes)} <= {4, 8}


def test_widest(tmp_path):
    """A launch has fewer than 2^32 threads along a dimension."""
    sizes = [(fp32, M, N, K) for fp32 in (False, True) for M in (1, 32) for N in (1, 1 << 20, (1 << 26) - 1, 1 << 26) for K in (1, 100, 10000, 1 << 27)]
    for (fp32, M, N, K), (columns, shares) in zip(sizes, choices(tmp_path, sizes)):
        assert columns in (1, 2, 4, 8) and 1 <= shares <= 64
        assert ((-(-N // (8 * columns)) + 7) // 8 * 8) * 1024 < 1 << 32
