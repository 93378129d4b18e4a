"""Host-side parts of the operators of residual networks, and what is said of their numerics, without a GPU."""
import os
import re

import numpy as np

from linear_tiles import PRODUCTS
from test_host_parts import ROOT, run_cpp


def nearest_bf16(x):
    bits = np.asarray(x, np.float32).view(np.uint32)
    return ((bits + ((bits >> 16) & 1) + 0x7fff) & 0xffff0000).astype(np.uint32).view(np.float32)


def thirds(x):
    h = nearest_bf16(x)
    m = nearest_bf16(x - h)
    l = (x - h) - m
    assert np.array_equal(nearest_bf16(l), l), "three bf16 numbers are all of an fp32 number"
    return [p.astype(np.float64) for p in (h, m, l)]


def test_what_fp32_products_leave_out():
    """The header's bound holds for random mantissas and for the worst ones, and is no more than twice what these take."""
    rng = np.random.default_rng(7)
    x, w = ((1 + rng.integers(0, 1 << 23, 1 << 20) / 2.0 ** 23).astype(np.float32) for _ in range(2))
    x[0] = w[0] = 1 + 2.0 ** -8 - 2.0 ** -17 - 2.0 ** -23
    (h, m, l), (_, m2, l2) = thirds(x), thirds(w)
    left = np.abs(m * l2 + l * m2 + l * l2) / (x.astype(np.float64) * w)
    said = re.search(r"Products of fp32 elements are exact to 2\^-(\d+)", open(os.path.join(ROOT, "include", "gcn.h")).read())
    bound = 2.0 ** -int(said.group(1))
    assert left.max() <= bound and left[0] > bound / 2


def test_launches_for_the_widest_rows_are_launchable(tmp_path):
    """Fewer than 2^32 threads along a dimension, and all columns in some workgroup, at the widths where these counts change and at the widest."""
    r = run_cpp(tmp_path, """
        #include <cstdio>
        #include <initializer_list>
        #include "launch_rules.h"
        using namespace gcn;
        int main() {
            const int64_t most = (int64_t)1 << 32;
            for (int64_t f : {int64_t(1), int64_t(16), int64_t(17), int64_t(1 << 20) - 1, int64_t(1 << 20), int64_t(1 << 20) + 1, int64_t(NORM_WIDEST) - 16,
                              int64_t(NORM_WIDEST) - 15, int64_t(NORM_WIDEST)}) {
                const LaunchGroups g = norm_vector_groups(f);
                if (g.x < 1 || g.y < 1 || g.x * int64_t(1024) >= most || g.y > 65535 || (int64_t)g.x * g.y * 16 < f)
                    return printf("norm vectors of %lld: %u x %u\\n", (long long)f, g.x, g.y), 1;
            }
            for (int64_t N : {int64_t(1), int64_t(64), int64_t(65), int64_t(LINEAR_WIDEST)}) {
                const int64_t groups = column_sum_groups(N);
                if (groups * 1024 >= most || groups * 64 < N) return printf("column sums of %lld\\n", (long long)N), 1;
            }
        }
    """)
    assert r.returncode == 0, r.stdout


def test_scratch_of_sums_over_the_rows(tmp_path):
    """Every row is in one share, and the partial sums of four vectors stay below 17 MB and four rows of fp32, for rows of any width."""
    r = run_cpp(tmp_path, """
        #include <cstdio>
        #include <initializer_list>
        #include "launch_rules.h"
        using namespace gcn;
        int main() {
            for (int64_t wide : {256, 512})
                for (int64_t f = 1; f <= NORM_WIDEST; f += f / 3 + 1)
                    for (int64_t n = 1; n <= 3000000; n += n / 2 + 1) {
                        const int64_t across = (f + wide - 1) / wide;
                        const RowShares s = row_shares(n, across, 256);
                        if (s.count < 1 || s.count > 65535 || s.rows % 4 || s.count * s.rows < n || (s.count - 1) * s.rows >= n)
                            return printf("shares of %lld rows\\n", (long long)n), 1;
                        if (s.count * f * 16 > 17000000 + 16 * f) return printf("%lld x %lld: %lld shares\\n", (long long)n, (long long)f, (long long)s.count), 1;
                    }
        }
    """)
    assert r.returncode == 0, r.stdout


def test_matrices_meet_where_they_have_a_byte_in_common(tmp_path):
    """Against the bytes of both, one by one: random matrices in a small buffer, contiguous and strided, at equal and at different pitches."""
    r = run_cpp(tmp_path, """
        #include <cstdio>
        #include <random>
        #include <set>
        #include "places.h"
        using namespace gcn;
        int main() {
            std::mt19937 rng(5);
            auto upto = [&](int n) { return (int)(rng() % (unsigned)(n + 1)); };
            static char buffer[4096];
            int met = 0, same = 0, between = 0;
            for (int round = 0; round < 200000; ++round) {
                struct M { int at, rows, cols, ld, bytes; } m[2];
                for (M& x : m) {
                    x.bytes = 2 << upto(1);
                    x.rows = 1 + upto(4); x.cols = 1 + upto(4); x.ld = x.cols + (upto(2) ? upto(6) : 0); x.at = 2 * upto(40);
                }
                if (upto(1)) { m[1].ld = m[0].ld < m[1].cols ? m[1].ld : m[0].ld; m[1].bytes = m[0].bytes; }
                if (!upto(9)) m[1] = m[0];
                std::set<int> have[2];
                for (int k = 0; k < 2; ++k)
                    for (int i = 0; i < m[k].rows; ++i)
                        for (int b = 0; b < m[k].cols * m[k].bytes; ++b) have[k].insert(m[k].at + i * m[k].ld * m[k].bytes + b);
                bool meet = false;
                for (int b : have[0]) meet |= have[1].count(b) > 0;
                const Span p(buffer + m[0].at, m[0].rows, m[0].cols, m[0].ld, m[0].bytes), q(buffer + m[1].at, m[1].rows, m[1].cols, m[1].ld, m[1].bytes);
                if (p.meets(q) != meet || q.meets(p) != meet) {
                    for (const M& x : m) printf("%d: %d x %d, %d apart, of %d bytes\\n", x.at, x.rows, x.cols, x.ld, x.bytes);
                    return 1;
                }
                if (m[0].rows == m[1].rows && m[0].bytes == m[1].bytes && p.is(q) != (have[0] == have[1] && m[0].cols == m[1].cols)) return printf("the same place\\n"), 1;
                met += meet; same += p.is(q);
                between += !meet && *have[0].begin() < *have[1].rbegin() && *have[1].begin() < *have[0].rbegin();
            }
            const Span none(nullptr, 3, 3, 3, 4), some(buffer, 3, 3, 3, 4);
            if (none.meets(some) || some.meets(none)) return printf("nothing meets something\\n"), 1;
            return met > 1000 && same > 1000 && between > 1000 ? 0 : (printf("%d %d %d\\n", met, same, between), 1);
        }
    """)
    assert r.returncode == 0, r.stdout


def test_every_tile_of_a_product_is_tested(tmp_path):
    """The sizes that the GPU tests take stand for the tile and the split that the rule gives them, and for all that there are."""
    for kind, whole, edge, splits, M, N, K in PRODUCTS:
        assert M % edge and N % edge and K % 64 and (not whole or (M % 8 == 0 and N % 8 == 0))
    calls = "".join(f'say({M}, {N}, {K}, {int(kind == "f32")}, {int(whole)});' for kind, whole, _, _, M, N, K in PRODUCTS)
    r = run_cpp(tmp_path, """
        #include <cstdio>
        #include "launch_rules.h"
        void say(int64_t M, int64_t N, int64_t K, int fp32, int direct) {
            const gcn::TileChoice c = gcn::choose_tiles(M, N, K, fp32, direct, 256);
            printf("%%d %%d\\n", c.edge, c.splits);
        }
        int main() { %s }
    """ % calls)
    assert [tuple(map(int, line.split())) for line in r.stdout.splitlines()] == [p[2:4] for p in PRODUCTS]
    assert {(p[0], p[1], p[2], p[3] > 1) for p in PRODUCTS} == {("16", w, e, s) for w in (False, True) for e in (256, 128, 64) for s in (False, True)} | {
        ("f32", False, e, s) for e in (128, 64) for s in (False, True)}
