"""The join at the top of the clipping's summation tree, compiled for the host: every count of values that a row
can have, against the tree padded with zeros, in an array of exactly the kernel's size between guards."""
import os
import re
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2402_11857_b200", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "balanced_join.h"
int main(int, char **argv) {   // argv: values, room; reads the values, prints the join and whether a guard was touched
    const int n = atoi(argv[1]), room = atoi(argv[2]);
    double s[4096];
    for (double &v : s) v = -1.0;
    for (int k = 0; k < n; ++k) if (scanf("%lf", &s[k]) != 1) return 1;
    const double r = liec::balanced_join(s, n);
    bool clean = true;
    for (int k = room; k < 4096; ++k) clean &= s[k] == -1.0;
    printf("%a %d\n", r, (int)clean);
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    where = tmp_path_factory.mktemp("join")
    (where / "join.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-O2", "-I", CSRC, str(where / "join.cpp"), "-o", str(where / "join")], check=True)
    return str(where / "join")


def room():
    text = open(os.path.join(CSRC, "clip_kernels.cu")).read()
    return int(re.search(r"constexpr int ROW_PASSES = (\d+);", text).group(1))


def padded_tree(values):
    s = np.asarray(values, np.float64)
    s = np.concatenate([s, np.zeros((1 << (len(s) - 1).bit_length()) - len(s))])
    while len(s) > 1:
        s = s[0::2] + s[1::2]
    return float(s[0])


# 145 passes of 4096 tiles: dim 2^32 - 1 in 65535 segments
@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 6, 7, 8, 9, 31, 33, 64, 65, 127, 128, 129, 143, 144, 145])
def test_any_count_within_the_array(program, n):
    values = np.random.default_rng(n).lognormal(0.0, 8.0, n)
    given = " ".join(float(v).hex() for v in values)
    out, clean = subprocess.run([program, str(n), str(room())], input=given, capture_output=True, text=True, check=True).stdout.split()
    assert float.fromhex(out) == padded_tree(values)
    assert clean == "1", "written beyond the kernel's array"
