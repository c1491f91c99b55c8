"""The rule by which the 4-bit attention's reference follows a row's largest score (csrc/cache4.hpp), compiled for the
host: a tile in which a score has grown is done again after the growth, so one growth has to end that, whatever the score.
"""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import paper_2608_20530_amd.build as B

SOURCE = """
#include "cache4.hpp"
using namespace lilicorr;
// growths until score x counts as known under reference m, as the kernel's loop does them (at most `most`); left: what the
// power's argument is then
extern "C" int growths(float x, float scale, float m, bool far, bool rule, int most, float* left) {
  int n = 0;
  far = far && rule;
  for (;; ++n) {
    const float s = far ? 1.f : scale, y = far ? scaled4(x, scale) : x;
    *left = fmaf(y, s, -m);
    if (!grown4(y, s, m) || n == most) return n;
    m = reference4(y, s);
    far = far || (rule && far4(m));
  }
}
"""


@pytest.fixture(scope="module")
def growths(tmp_path_factory):
    d = tmp_path_factory.mktemp("rule")
    source = d / "rule.hip"
    source.write_text(SOURCE)
    flags = [f for f in B.FLAGS if f != "-Wall"] + ["--offload-host-only", "-w"]
    subprocess.run(["hipcc", *flags, "-I", os.path.join(B.ROOT, "include"), "-I", B.CSRC, "-o", str(d / "rule.so"), str(source)],
                   check=True)
    f = ctypes.CDLL(str(d / "rule.so")).growths
    f.argtypes = [ctypes.c_float] * 3 + [ctypes.c_bool] * 2 + [ctypes.c_int, ctypes.POINTER(ctypes.c_float)]
    left = ctypes.c_float()

    def call(x, scale, m=-np.inf, far=False, rule=True, most=5):
        return f(float(x), float(scale), float(m), far, rule, most, ctypes.byref(left)), left.value
    return call


SCALES = [np.float32(1.4426950408889634 / np.sqrt(d)) for d in (32, 64, 96, 128, 256)] + [1.0, 0.37, 3.1, 1e-9, 2.0 ** 40]


@pytest.mark.parametrize("scale", SCALES)
def test_a_far_neighbour(growths, scale):
    """Another row's reference goes far: products are rounded from then on. A row that needed no growth, or has had one, needs
    one more at most."""
    g = np.random.default_rng(2)
    for e in range(-20, 24):
        for m in np.floor(g.uniform(-1, 1, 50) * 2.0 ** e):
            x = np.float32((m + g.uniform(-20, 20)) / scale)
            n, left = growths(x, scale, m, far=True)
            assert n <= 1 and not left > 8, (x, scale, m, left)


@pytest.mark.parametrize("scale", SCALES)
def test_one_growth_is_enough(growths, scale):
    g = np.random.default_rng(1)
    with np.errstate(over="ignore"):
        x = np.concatenate([np.float32(s * g.uniform(1, 2, 40)) * np.float32(2.0 ** e) for e in range(-126, 128) for s in (1, -1)])
    for m, far in ((-np.inf, False), (-np.inf, True), (0.0, False), (-(2.0 ** 24) + 1, False), (2.0 ** 30, True), (-(2.0 ** 100), True)):
        for v in x:
            n, left = growths(v, scale, m, far)
            assert n <= 1 and not left > 8, (v, scale, m, far, n, left)
            if n and abs(np.float64(v) * scale) < 3e38:
                assert -2 < left < 2, (v, scale, m, far, left)  # the power of the largest score counts


def test_values_that_are_no_scores(growths):
    for scale in SCALES:
        for m, far in ((-np.inf, False), (5.0, False), (2.0 ** 40, True), (np.inf, True)):
            for v in (np.inf, -np.inf, np.nan):
                assert growths(v, scale, m, far)[0] <= 1


def test_rounding_alone_would_never_end(growths):
    """Heads of 128, queries of 20480 or 168 and keys of 6144 or 98304 throughout: without the second form the same
    reference comes back."""
    for q, k in ((20480, 6144), (168, 6 * 2 ** 14)):
        x, scale = np.float32(128 * q * k), np.float32(1.4426950408889634 / np.sqrt(128))
        assert growths(x, scale, rule=False, most=50)[0] == 50 and growths(x, scale)[0] == 1
