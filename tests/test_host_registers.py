"""Registers of the linear layers' kernels as the compiler gave them: what a change beside a kernel takes from it shows here, and not in its results.  Read from the built library, so without a GPU."""
import os
import re

import pytest

pytest.importorskip("msgpack")

import kernel_registers
from paper_2005_03300_amd import build

TYPES = {"DF16b": "bf16", "DF16_": "f16"}
WAYS = {(0, 1): "forward", (0, 0): "dX", (1, 1): "dW"}


@pytest.fixture(scope="module")
def kernels():
    if not os.path.exists(build.LIB):
        build.build()
    return kernel_registers.kernels(build.LIB)


def test_spilled_registers_of_linear_layers(kernels):
    """The 256 x 256 tile through registers holds all there are and spills some; no other tile of 16-bit elements spills a vector register."""
    most = {("bf16", "forward"): (23, 18), ("f16", "forward"): (19, 18), ("bf16", "dX"): (0, 0), ("f16", "dX"): (0, 0), ("bf16", "dW"): (60, 0), ("f16", "dW"): (78, 0)}
    seen = 0
    for name, k in kernels.items():
        m = re.match(r"_ZN3gcn13k_linear_tileI(DF16b|DF16_)Li(\d+)ELi\d+ELi\d+ELi\d+ELi(\d)ELi(\d)ELb(\d)ELb0EEE", name)
        if not m:
            continue
        seen += 1
        type_, edge, way, direct = TYPES[m[1]], int(m[2]), WAYS[int(m[3]), int(m[4])], m[5] == "1"
        vector, scalar = most[type_, way] if edge == 256 and not direct else (0, 28)
        assert k[".vgpr_spill_count"] <= vector and k[".sgpr_spill_count"] <= scalar, (name, k[".vgpr_spill_count"], k[".sgpr_spill_count"])
    assert seen == 36


def test_registers_of_linear_slopes(kernels):
    """The elementwise pass with two rows ahead leaves room for eight wavefronts on a SIMD (16-bit elements: seven); nothing of it is spilled."""
    most = {"f": 64, "DF16b": 72, "DF16_": 72}
    seen = 0
    for name, k in kernels.items():
        m = re.match(r"_ZN3gcn14k_linear_slopeI(f|DF16b|DF16_)Li(\d)ELb(\d)EEE", name)
        if not m:
            continue
        seen += 1
        assert k[".vgpr_spill_count"] == k[".sgpr_spill_count"] == 0, name
        if m[2] == "2" and m[3] == "1":
            assert k[".vgpr_count"] <= most[m[1]], (name, k[".vgpr_count"])
    assert seen == 12


def test_rows_ahead(tmp_path):
    """Two rows ahead for short shares, and for rows of 16 KB whose shares begin 2 MB apart."""
    from test_host_parts import run_cpp
    cases = [(4, 2048, 2), (16, 2048, 2), (20, 8192, 2), (28, 602, 2), (32, 4096, 4), (64, 1024, 4), (228, 256, 4), (128, 16384, 2), (256, 32768, 2), (68, 16384, 4), (256, 8192, 4), (128, 16386, 4)]
    r = run_cpp(tmp_path, '''
        #include <cstdio>
        #include "launch_rules.h"
        int main() { %s }
    ''' % "".join(f'printf("%d ", gcn::slope_rows_ahead({a}, {b}));' for a, b, _ in cases))
    assert list(map(int, r.stdout.split())) == [w for _, _, w in cases]


def test_sizes_take_the_slopes_that_they_stand_for(tmp_path):
    from linear_slopes import SLOPES
    from test_host_parts import run_cpp
    r = run_cpp(tmp_path, '''
        #include <cstdio>
        #include "launch_rules.h"
        static void size(int64_t n, int64_t N, int64_t bytes) {
            const int64_t wide = 64 * (16 / bytes), across = (N + wide - 1) / wide;
            printf("%%d %%d\\n", gcn::slope_rows_ahead(gcn::row_shares(n, across, 256).rows, N * bytes), N %% (16 / bytes) == 0);
        }
        int main() { %s }
    ''' % "".join(f"size({n}, {N}, {4 if t == 'f32' else 2});" for t, _, _, n, N in SLOPES))
    got = [(int(a), b == "1") for a, b in map(str.split, r.stdout.splitlines())]
    assert got == [p[1:3] for p in SLOPES], [(p, q) for p, q in zip(SLOPES, got) if p[1:3] != q]
    assert {p[:3] for p in SLOPES} == {(t, a, w) for t in ("16", "f32") for a in (2, 4) for w in (False, True)}
