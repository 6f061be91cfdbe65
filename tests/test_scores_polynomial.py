"""The polynomial that stands for the tanh of a capped score where the products are small enough (csrc/scoring.h): the constants that the host
hands to the kernels, built and run on the CPU, and the kernels' steps with them in float32, against tanh in 64 bits."""
import os
import subprocess

import numpy as np
import pytest

from paper_2411_09909_amd import build

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "%s/scoring.h"
int main(int argc, char** argv) {
  for (int i = 1; i + 1 < argc; i += 2) {
    const amx_scores_t s = {strtof(argv[i], nullptr), 0, nullptr};
    const amx::Scores r = amx::scores_of(&s, strtof(argv[i + 1], nullptr));
    printf("%%a %%a %%a %%a %%a %%a\n", r.scale, r.small, r.k1, r.k2, r.k3, r.k4);
  }
}
"""
CASES = [(2.0 ** c, 2.0 ** s) for c in (-20, -7, 0, 5, 13, 20) for s in (-149, -126, -100, -97, -90, -80, -60, -45, -33, -20, -10, -3, 0, 9, 19, 25, 99)]


@pytest.fixture(scope="module")
def scores_of(tmp_path_factory):
    at = tmp_path_factory.mktemp("scores")
    source, program = str(at / "scores.hip"), str(at / "scores")
    with open(source, "w") as f:
        f.write(PROGRAM % build.CSRC)
    subprocess.run(["hipcc", "--offload-arch=gfx950", "-std=c++20", "-O1", source, "-o", program], check=True, capture_output=True, text=True, timeout=300)
    out = subprocess.run([program] + [float.hex(v) for c in CASES for v in c], check=True, capture_output=True, text=True, timeout=60,
                         env={**os.environ, "HIP_VISIBLE_DEVICES": ""}).stdout
    rows = [[float.fromhex(v) for v in line.split()] for line in out.splitlines()]
    assert len(rows) == len(CASES)
    return rows


def test_the_polynomial_over_all_products_it_may_take(scores_of):
    """The fit's 2^-27.4 and, of the roundings of 2^-24, those of the scale (two), of the last sum and of the last product whole and of the rest some fifth: below
    2^-22 of the score (some more here, where products and sums round apart: 2^-21.7). What is lost where a power of a constant leaves FP32's range is
    below 2^-126 times a product of at most 2^60, and the scale of such a call as much of the cap: 2^-40 of that."""
    f = np.float32
    for (cap, scale), (first, small, k1, k2, k3, k4) in zip(CASES, scores_of):
        if small == 0:
            continue
        assert np.isfinite([first, small, k1, k2, k3, k4]).all(), (cap, scale)
        s = np.concatenate([[0.0], np.exp2(np.arange(-60.0, 128.0, 0.25)), [small, 0.999 * small]])
        s = s[s <= small].astype(f)
        with np.errstate(over="ignore", invalid="ignore", under="ignore"):
            u = s * s
            p = (u * f(k4) + f(k3)).astype(f)
            p = (u * p + f(k2)).astype(f)
            p = (u * p + f(k1)).astype(f)
            p = (u * p + f(first)).astype(f)
            got = (s * p).astype(np.float64)
        want = cap * np.tanh(s.astype(np.float64) * scale / cap) * np.log2(np.e)
        assert np.isfinite(got).all(), "cap %g, scale %g: products from %g on" % (cap, scale, s[~np.isfinite(got)].min())
        assert (np.abs(got - want) <= 2.0 ** -21.7 * np.abs(want) + 2.0 ** -40 * cap).all(), (cap, scale)
