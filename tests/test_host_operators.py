"""Host-side parts of the operators of residual networks, and what is said of their numerics, without a GPU."""
import os
import re

import numpy as np

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
