"""The attention kernels' softmax arithmetic (csrc/softmax_rule.cuh) on the CPU: rows of finite scores of any size keep finite sums that
are not 0, and the block kernel's loop that raises a maximum ends.

``row`` walks a row of scores as the block kernel does: the maximum of the first 128, then halves of a tile (64 scores), whose sum may raise it.
It counts the passes over a half.  With ``planted`` the maximum is scaled and rounded, the product with the scale is not, as in one
multiply-add, and the count of raises is not looked at: that must be seen to go round without an end (the driver stops it)."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2509_23410_b200", "csrc")

DRIVER = r"""
#include "softmax_rule.cuh"
#include <math.h>
using namespace patch::attn;
static float top_of(const float* s, int n) {
    float t = -INFINITY;
    for (int i = 0; i < n; ++i) t = fmaxf(t, s[i]);
    return t;
}
// out: maximum, sum, largest sum of a half as it was taken; returns the most passes over a half
extern "C" int row(const float* s, int n, float scale, int planted, float* out) {
    float m = top_of(s, 128), l = 0.0f, most = 0.0f;
    int passes = 0;
    for (int h = 0; h < n; h += 64) {
        bool raised = false;
        for (int pass = 1;; ++pass, raised = true) {
            float sum = 0.0f;
            for (int i = h; i < h + 64; ++i)
                sum += exp2f(planted ? fmaf(s[i], scale, -(base_of(m) * scale)) : exponent(s[i], base_of(m), scale));
            if (pass > passes) passes = pass;
            if (!raise_maximum(sum, m, raised && !planted) || pass == 50) {
                l += sum;
                if (sum > most) most = sum;
                break;
            }
            const float up = fmaxf(m, top_of(s + h, 64)), a = up == -INFINITY ? 1.0f : exp2f(exponent(m, up, scale));
            m = up;
            l *= a;
        }
    }
    out[0] = m; out[1] = l; out[2] = most;
    return passes;
}
"""


@pytest.fixture(scope="module")
def row(tmp_path_factory):
    d = tmp_path_factory.mktemp("rule")
    (d / "driver.cpp").write_text(DRIVER)
    so = str(d / "driver.so")
    subprocess.run(["g++", "-O2", "-std=c++17", "-ffp-contract=off", "-fPIC", "-shared", f"-I{CSRC}", str(d / "driver.cpp"), "-o", so], check=True)
    f = ctypes.CDLL(so).row
    f.restype = ctypes.c_int
    f.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_int, ctypes.c_void_p]

    def call(s, scale, planted=False):
        s, out = np.ascontiguousarray(s, np.float32), np.zeros(3, np.float32)
        return f(s.ctypes.data, len(s), scale, planted, out.ctypes.data), *map(float, out)
    return call


SCALES = [np.float32(128 ** -0.5 * 1.4426950408889634), np.float32(64 ** -0.5 * 1.4426950408889634), np.float32(0.37 * 1.4426950408889634)]


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("power", list(range(-4, 44, 2)) + [60, 90, 120])
def test_rows_of_any_size(row, scale, power):
    """The largest probability is exactly 1 in the half that holds it, so the sum lies between what is left of 1 and the number of keys."""
    rng = np.random.default_rng(power + 100)
    for i in range(40):
        s = (rng.standard_normal(512) * np.float32(2.0) ** power).astype(np.float32)
        if i % 4 == 1:
            s = np.sort(s)                     # ever larger: the maximum is raised again and again
        if i % 4 == 2:
            s = -np.abs(s) - np.float32(2.0) ** power
        if i % 4 == 3:
            s[:128] = -np.abs(s[:128])
        passes, m, l, most = row(s, scale)
        assert passes <= 2
        assert m <= s.max() and np.isfinite(l) and l > 0.0
        assert most <= 256.0 + 64.0
        # against the definition in 64 bits: 512 additions and rescalings in fp32, exp2f good to 2^-22, an exponent x of two roundings (what
        # is summed to more than 256 is taken anew, so x is at most 8 and below -150 the probability is 0: 2^-23 150 ln 2)
        want = np.exp2((s.astype(np.float64) - m) * np.float64(scale)).sum()
        assert abs(l - want) <= want * 2.0 ** -13


@pytest.mark.parametrize("scale", SCALES)
def test_rows_with_masked_scores(row, scale):
    s = np.full(256, -np.inf, np.float32)
    assert row(s, scale)[1:3] == (-np.inf, 0.0)
    s[3] = -3e38
    passes, m, l, _ = row(s, scale)
    assert passes == 1 and np.isfinite(m) and l == 1.0


def test_the_loop_ends_for_infinite_scores(row):
    s = np.zeros(512, np.float32)
    s[200] = np.inf
    assert row(s, SCALES[0])[0] <= 2
    s[5] = np.inf
    assert row(s, SCALES[0])[0] == 1
    s[7] = np.nan
    assert row(s, SCALES[0])[0] == 1


def test_a_planted_mistake_is_seen(row):
    """An unrounded product against a rounded one: rows of this size go round for ever, larger ones also vanish."""
    rng = np.random.default_rng(1)
    endless = vanished = 0
    for power in (31, 33, 36):
        for _ in range(40):
            s = (rng.standard_normal(512) * 2.0 ** power).astype(np.float32)
            passes, _, l, _ = row(s, SCALES[0], planted=True)
            endless += passes == 50
            vanished += l == 0.0
    assert endless and vanished
