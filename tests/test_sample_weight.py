"""The weight of a logit in sample.cu, 2^-(c (top - v)) as a whole number of 2^-44, from the kernel's own header compiled by g++ against
64 bits; no GPU is needed.

A weight is m 2^-30 shifted right.  m is the table's entry e (2^29 to 2^30, off by half a step) and a correction of up to 2^21.5 steps from
a series cut off under 2^-38 of the weight (half a step again for its rounding, 0.2 for that of its float product); c in two floats is
off by 2^-48 of itself, which is 45 2^-48 of y and 2^-43 of the weight, and y_low by 2^-42.  Together under 1.5 steps of 2^-30 where
e is 2^29 at least: 2^-28.4 of the weight, and a step of 2^-44 is cut off by the shift."""
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2410_05911_gb300", "csrc")

HARNESS = r"""
#include "sample_weight.cuh"
#include <cstdio>
#include <vector>
static const aecct::PowerTable table;
int main() {
  float x[5];
  while (std::fread(x, 4, 5, stdin) == 5) {
    const uint64_t w = aecct::weight_of(x[1], x[0], x[2], x[3], x[4], [](uint32_t j) { return table.e[j]; });
    std::fwrite(&w, 8, 1, stdout);
  }
  return 0;
}
"""
TYPES = ["float32", "float16", "bfloat16"]


@pytest.fixture(scope="module")
def harness(tmp_path_factory):
    d = tmp_path_factory.mktemp("sample_weight")
    src, exe = d / "harness.cpp", d / "harness"
    src.write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-O1", "-ffp-contract=off", f"-I{CSRC}", str(src), "-o", str(exe)], check=True)
    return str(exe)


def rounded(x, dtype):
    x = np.asarray(x, np.float64)
    if dtype == "float16":
        return x.astype(np.float16).astype(np.float32)
    x = x.astype(np.float32)
    if dtype == "bfloat16":
        bits = x.view(np.uint32)
        x = ((bits + 0x7FFF + ((bits >> 16) & 1)) & np.uint32(0xFFFF0000)).view(np.float32)
    return x


def weights(harness, top, v, t):
    """The kernel's weights, and the definition's in units of 2^-44."""
    top, v, t = (np.asarray(a, np.float32) for a in np.broadcast_arrays(top, v, t))
    c64 = 1.4426950408889634074 / t.astype(np.float64)
    c = c64.astype(np.float32)
    low = (c64 - c).astype(np.float32)
    off = (45.0 / c.astype(np.float64)).astype(np.float32)  # (rounded down)
    off = np.where(off.astype(np.float64) * c > 45.0, np.nextafter(off, np.float32(0)), off)
    records = np.stack([top, v, c, low, off], 1).astype(np.float32)
    out = subprocess.run([harness], input=records.tobytes(), capture_output=True, check=True).stdout
    with np.errstate(invalid="ignore", over="ignore", under="ignore"):
        d = np.where(top == v, 0.0, top.astype(np.float64) - v)
        want = 2.0 ** 44 * np.exp2(-c64 * d)
    return np.frombuffer(out, np.uint64).astype(np.float64), want


def check(got, want):
    off = np.abs(got - want) - (2.0 ** -28 * want + 1)
    assert (off <= 0).all(), (int(off.argmax()), off.max(), (np.abs(got - want) / np.maximum(want, 1)).max())


@pytest.mark.parametrize("dtype", TYPES)
def test_logits_of_every_size(harness, dtype):
    r = np.random.default_rng(1)
    n = 200_000
    top = rounded(r.choice([-1, 1], n) * np.exp2(r.uniform(-8, 6, n)), dtype)
    t = np.exp2(r.uniform(-3, 5, n)).astype(np.float32)
    near = top - rounded(t * r.uniform(0, 31, n), dtype)  # 45 octaves under the largest
    tiny = r.choice([-1, 1], n) * np.exp2(r.uniform(-24, -4, n))  # far from the largest in size
    v = np.minimum(rounded(np.where(r.random(n) < 0.5, near, tiny), dtype), top)
    check(*weights(harness, top, v, t))


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_small_logits_under_a_large_one(harness, dtype):
    """top - v does not fit 24 bits: what its rounding leaves out counts."""
    r = np.random.default_rng(2)
    v = rounded(r.choice([-1, 1], 20_000) * np.exp2(r.uniform(-24, -10, 20_000)), dtype)
    for top in (2.0, 8.0, 20.0):
        for t in (0.5, 0.7, 1.0, 3.0):
            check(*weights(harness, top, v, t))


@pytest.mark.parametrize("dtype", TYPES)
def test_large_logits_under_a_small_one(harness, dtype):
    """Temperatures so high that logits of 2^16 times the largest one's size count."""
    r = np.random.default_rng(3)
    top = rounded(r.choice([-1, 1], 20_000) * np.exp2(r.uniform(-12, -2, 20_000)), dtype)
    v = rounded(-np.exp2(r.uniform(8, 15.9, 20_000)), dtype)
    check(*weights(harness, top, v, 2.0 ** 15))
    check(*weights(harness, top, v, 3e4))


@pytest.mark.parametrize("dtype", TYPES)
def test_temperatures_at_the_ends(harness, dtype):
    v = rounded([1.0, 1.0 - 2.0 ** -7, 0.5, 0.0, -1.0, -6e4], dtype)
    for t in (2.0 ** -100, 2.0 ** -20, 2.0 ** 40, 2.0 ** 100):
        check(*weights(harness, v[0], v, t))


@pytest.mark.parametrize("dtype", TYPES)
def test_the_largest_logit_weighs_one(harness, dtype):
    for top in (0.0, -0.0, 1.0, -1e4, 3e4):
        got, _ = weights(harness, rounded(top, dtype), rounded(top, dtype), [0.3, 1.0, 7.0])
        assert (got == 2.0 ** 44).all()
    got, _ = weights(harness, 1.0, -np.inf, [0.3, 1.0, 7.0])
    assert not got.any()


def test_infinity_under_itself_weighs_one(harness):
    got, _ = weights(harness, np.inf, np.inf, [2.0 ** -100, 0.3, 1.0, 7.0, 2.0 ** 100])
    assert (got == 2.0 ** 44).all(), got / 2.0 ** 44
    for v in (-np.inf, -3e38, 0.0, 3e38):
        got, _ = weights(harness, np.inf, v, [2.0 ** -100, 0.3, 1.0, 7.0, 2.0 ** 100])
        assert not got.any()
